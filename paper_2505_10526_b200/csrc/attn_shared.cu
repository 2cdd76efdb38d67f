// Verify attention of sequences whose contexts begin with the same positions (massv_verify_attn_shared).
//
// softmax over positions [0, L + j] is the merge of softmax over a shared prefix [0, s) and over the rest: with m the maximum,
// l the sum and O the weighted values of each part relative to its m,
//   out = (O_1 2^(m_1 - m) + O_2 2^(m_2 - m)) / (l_1 2^(m_1 - m) + l_2 2^(m_2 - m)),   m = max(m_1, m_2).
// The rest of every sequence goes through the kernels of massv_verify_attn, on page tables and lengths shifted by s
// (attn_tail_kernel writes them; causality only depends on differences of positions).  The prefix is read once per group:
// the rows of all its sequences stand together, so that what was a stream of bytes per sequence becomes a matrix product of hundreds
// to thousands of rows with the prefix, on tcgen05:
//
//   S[128, 128] = Q[128 rows, d] K_block^T          Q and K in shared memory as TMA writes them, S in tensor memory
//   P           = 2^(S scale log2 e - reference)    one row per thread; bf16, back into the columns of S
//   O[128, d]  += P[128, 128] V_block               P read from tensor memory, V from shared memory
//
// A tile is as many whole (sequence, block row) pairs of a KV head's G query heads as fit 128 rows.  At head_dim 64 and 128 a CTA
// works on two tiles at once, so that one tile's products run under the other's exponentials; both share each K and V block.  At 256
// the accumulator leaves room for one, whose scores are double buffered instead: the scores of the next block are formed under
// the exponentials of this one.  Warp 0 copies (TMA), one thread of warp 1 issues the products, four warps per tile make the softmax.
// Every position of the prefix is seen by every row: there is nothing to mask.
//
// The (group, tiles, KV head, block) products form one line, cut into equal ranges for a persistent grid of one CTA per SM.
// Tiles inside one range are merged with the rest and written at once; those that a cut divides leave
// pieces to attn_prefix_merge_kernel.
#include "kernels.cuh"
#include "ptx.cuh"
#include "umma.cuh"

namespace massv {

namespace {

constexpr int kTileRows = 128;
constexpr int kPagesPerBlock = kPrefixBlock / kPageSize;
constexpr float kRescaleThreshold = 8.f;   // log2 units a row's maximum may outgrow its reference by

template <int D>
struct PrefixCfg {
    static constexpr int kTiles = D == 256 ? 1 : 2;           // query tiles of a CTA
    static constexpr int kParts = D == 256 ? 2 : 1;           // ring entries of a K block (halves of d) and of a V block (halves of the positions)
    static constexpr int kNCH = D / 64;
    static constexpr int kQTile = kTileRows * D * 2;
    static constexpr int kEntry = kPrefixBlock * D * 2 / kParts;
    static constexpr int kEntries = D == 64 ? 8 : 5;
    static constexpr int kBoxes = kPagesPerBlock * kNCH / kParts;      // 16-position x 64-element boxes of an entry
    static constexpr int kSmem = kTiles * kQTile + kEntries * kEntry + 1024;
    static constexpr int kThreads = 128 + kTiles * 128;
    static constexpr uint32_t kTmemCols = 512;
    static constexpr uint32_t kTmemO = 2 * kPrefixBlock;      // two score buffers, then the accumulators
    static_assert(kBoxes <= 32 && kTmemO + kTiles * D <= kTmemCols && kSmem <= 226 * 1024, "fits");
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

// ---- groups, and the page tables and lengths of what the sequences do not share.  One CTA per sequence.
__global__ void __launch_bounds__(128) attn_tail_kernel(const SharedAttnParams p) {
    const int b = blockIdx.x, t = threadIdx.x, R = p.a.R, cap = p.a.max_pages * kPageSize;
    __shared__ int s_bad, s_group, s_min, s_src, s_members;
    if (t == 0) { s_bad = 0; s_group = 0; s_min = 0x7fffffff; s_src = 0x7fffffff; s_members = 0; }
    pdl_wait();
    pdl_trigger();
    __syncthreads();
    for (int i = t; i < p.n_groups; i += blockDim.x) {
        const int lo = p.group_start[i], hi = p.group_start[i + 1];
        if (lo > hi || (i == 0 && lo != 0) || (i == p.n_groups - 1 && hi != p.a.B)) s_bad = 1;
        if (lo <= b && b < hi) s_group = i;
    }
    __syncthreads();
    const bool bad = s_bad != 0;
    const int g = s_group, lo = bad ? b : p.group_start[g], hi = bad ? b + 1 : p.group_start[g + 1];
    auto fits = [&](int L) { return L >= 0 && L + R <= cap; };
    for (int m = lo + t; m < hi; m += blockDim.x) {
        const int L = p.a.seq_lens[m];
        if (!fits(L)) continue;                        // (the kernels of the rest skip and report it)
        atomicMin(&s_min, L);
        atomicMin(&s_src, m);
        atomicAdd(&s_members, 1);
    }
    __syncthreads();
    // whole blocks that every member has committed; a sequence alone shares nothing
    const int blocks = bad || s_members < 2 ? 0 : max(0, min(p.shared_lens[g], s_min)) / kPrefixBlock;
    if (bad && b == 0 && t == 0) set_status(p.a.dev_status, MASSV_ERR_INVALID_ARG);
    if (!bad && b == lo && t == 0) p.groups[g] = make_int4(blocks, s_src, lo * R, (hi - lo) * R);
    if (b == 0)
        for (int i = t; i < p.n_groups; i += blockDim.x)
            if (bad || p.group_start[i] == p.group_start[i + 1]) p.groups[i] = make_int4(0, 0, 0, 0);
    const int L = p.a.seq_lens[b];
    const bool ok = fits(L);
    const int skip = ok ? blocks * kPrefixBlock : 0;
    if (t == 0) { p.skip[b] = skip; p.tail_lens[b] = L - skip; }
    if (!ok) return;
    const int32_t* src = p.a.page_table + (size_t)b * p.a.max_pages;
    int32_t* dst = p.tail_table + (size_t)b * p.a.max_pages;
    const int first = skip / kPageSize, n = (L + R + kPageSize - 1) / kPageSize;
    for (int i = first + t; i < n; i += blockDim.x) dst[i - first] = src[i];
}

// A run of blocks of one (group, tiles, KV head).
struct PrefixSeg {
    int head, src;
    int blk0;            // first (sequence, block row) pair of the first tile
    int n_rows[2];       // query rows of each tile
    int kb0, n;          // blocks
    int whole;           // every block of the prefix: no piece
    int slot;
};

// Where unit u of the line lies.
struct PrefixItem { int g, blocks, tile, head, kb, start; };

__device__ __forceinline__ PrefixItem prefix_item(const SharedAttnParams& p, const int* cum, int u) {
    int lo = 0, hi = p.n_groups - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (cum[mid] <= u) lo = mid; else hi = mid - 1;
    }
    PrefixItem it;
    it.g = lo;
    it.blocks = p.groups[lo].x;
    const int off = u - cum[lo], item = off / it.blocks;
    it.kb = off - item * it.blocks;
    it.tile = item / p.a.Hkv;
    it.head = item - it.tile * p.a.Hkv;
    it.start = u - it.kb;
    return it;
}

template <int D>
__global__ void __launch_bounds__(PrefixCfg<D>::kThreads, 1)
attn_prefix_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_q,
                   const SharedAttnParams p) {
    using Cfg = PrefixCfg<D>;
    constexpr int E = Cfg::kEntries, NT = Cfg::kTiles, PARTS = Cfg::kParts, NCH = Cfg::kNCH;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t ready_bar[E], empty_bar[E];
    __shared__ __align__(8) uint64_t q_ready_bar, q_free_bar;
    __shared__ __align__(8) uint64_t s_full_bar[2], p_full_bar[2];     // by score buffer
    __shared__ __align__(8) uint64_t o_full_bar[2], o_free_bar[2];     // by tile
    __shared__ __align__(8) uint64_t pv_done_bar;                      // one tile: O is up to date
    __shared__ int s_cum[kMaxGroups + 1];
    __shared__ uint32_t tmem_base_slot;
    __shared__ int abort_flag;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int G = p.a.Hq / p.a.Hkv, nb = kTileRows / G, tile_rows = nb * G;
    if (threadIdx.x == 0) {
        for (int e = 0; e < E; ++e) { mbar_init(&ready_bar[e], 1); mbar_init(&empty_bar[e], 1); }
        mbar_init(&q_ready_bar, 1); mbar_init(&q_free_bar, 1); mbar_init(&pv_done_bar, 1);
        for (int i = 0; i < 2; ++i) { mbar_init(&s_full_bar[i], 1); mbar_init(&p_full_bar[i], 4); mbar_init(&o_full_bar[i], 1); mbar_init(&o_free_bar[i], 4); }
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        __syncwarp();
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base_slot)), "r"(Cfg::kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    pdl_wait();

    // ---- the line: units of group 0 .. g-1
    for (int i = threadIdx.x; i < p.n_groups; i += blockDim.x) {
        const int4 gr = p.groups[i];
        s_cum[i + 1] = (gr.w + nb * NT - 1) / (nb * NT) * p.a.Hkv * gr.x;
    }
    if (threadIdx.x == 0) s_cum[0] = 0;
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* q_smem = smem + E * Cfg::kEntry;                          // [tile][d / 64][128 rows][128 B], swizzled
    // rows past the last pair of a tile are never copied
    for (int i = threadIdx.x; i < NT * NCH * (kTileRows - tile_rows) * 8; i += blockDim.x) {
        const int per = (kTileRows - tile_rows) * 8, region = i / per, k = i - region * per;
        *reinterpret_cast<uint4*>(q_smem + region * (kTileRows * 128) + tile_rows * 128 + k * 16) = make_uint4(0u, 0u, 0u, 0u);
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncthreads();
    if (warp == 0) {
        int run = 0;
        for (int i0 = 0; i0 < p.n_groups; i0 += 32) {
            const int i = i0 + lane;
            int incl = i < p.n_groups ? s_cum[i + 1] : 0;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int v = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += v;
            }
            if (i < p.n_groups) s_cum[i + 1] = run + incl;
            run += __shfl_sync(0xffffffffu, incl, 31);
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const int total = s_cum[p.n_groups];
    const int per_cta = max(1, (total + (int)gridDim.x - 1) / (int)gridDim.x);
    if (blockIdx.x == 0) {
        for (int i = threadIdx.x; i <= p.n_groups; i += blockDim.x) p.meta[1 + i] = s_cum[i];
        if (threadIdx.x == 0) p.meta[0] = per_cta;
    }
    const int f_first = min(total, (int)blockIdx.x * per_cta), f_end = min(total, f_first + per_cta);
    int f = f_first;
    auto next_segment = [&](PrefixSeg& sg) -> bool {
        if (f >= f_end) return false;
        const PrefixItem it = prefix_item(p, s_cum, f);
        const int4 gr = p.groups[it.g];
        sg.head = it.head; sg.src = gr.y;
        const int done = it.tile * nb * NT;                            // pairs of earlier tiles
        sg.blk0 = gr.z + done;
        sg.n_rows[0] = min(nb, gr.w - done) * G;
        sg.n_rows[1] = NT == 2 ? max(0, min(nb, gr.w - done - nb)) * G : 0;
        sg.kb0 = it.kb;
        sg.n = min(it.blocks - it.kb, f_end - f);
        sg.whole = sg.n == it.blocks;
        // slot 0: the piece that opens this CTA's range; slot 1: one that runs on into the next CTA's
        sg.slot = (int)blockIdx.x * 2 + (f == f_first ? 0 : 1);
        f += sg.n;
        return true;
    };

    const uint32_t tmem_base = tmem_base_slot;
    volatile int* abort_ptr = &abort_flag;
    PrefixSeg sg;
    if (f >= f_end) {
        // nothing to compute: fall through to the release of tensor memory
    } else if (warp == 0) {
        // ------------------------------------------------ copies
        uint64_t policy;
        asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(policy));
        int it = 0;                      // entries filled so far
        bool ok = true;
        for (int seg = 0; ok && next_segment(sg); ++seg) {
            if (seg >= 1) {
                int fr = 0;
                if (lane == 0) fr = mbar_wait(&q_free_bar, (uint32_t)(seg - 1) & 1u, abort_ptr) ? 1 : 0;
                if (!__shfl_sync(0xffffffffu, fr, 0)) { ok = false; break; }
            }
            const int tiles = sg.n_rows[1] > 0 ? 2 : 1;
            if (lane == 0) mbar_expect_tx(&q_ready_bar, (uint32_t)(tiles * tile_rows * D * 2));
            __syncwarp();
            if (lane < tiles * NCH) {
                const int x = lane / NCH, dc = lane % NCH;
                tma_load_3d(q_smem + x * Cfg::kQTile + dc * (kTileRows * 128), &map_q, dc * 64, sg.head * G, sg.blk0 + x * nb, &q_ready_bar, policy);
            }
            // page ids travel in registers: lane l holds page 32 * group + l of the segment, four blocks to a group
            const int32_t* pt = p.a.page_table + (size_t)sg.src * p.a.max_pages + sg.kb0 * kPagesPerBlock;
            const int n_pages = sg.n * kPagesPerBlock;
            int pid_prev = 0, pid_cur = lane < n_pages ? pt[lane] : 0, pid_next = 32 + lane < n_pages ? pt[32 + lane] : 0, grp = 0;
            for (int i = 0; i < 2 * sg.n && ok; ++i) {
                int t, is_v;             // in the order in which the products take them
                if (NT == 2) { t = i >> 1; is_v = i & 1; }
                else if (i == 0) { t = 0; is_v = 0; }
                else if (i == 2 * sg.n - 1) { t = sg.n - 1; is_v = 1; }
                else if (i & 1) { t = (i + 1) >> 1; is_v = 0; }
                else { t = (i >> 1) - 1; is_v = 1; }
                if (t / 4 > grp) {       // only a K block can be the first of a new group
                    grp = t / 4;
                    pid_prev = pid_cur; pid_cur = pid_next;
                    const int nxt = (grp + 1) * 32 + lane;
                    pid_next = nxt < n_pages ? pt[nxt] : 0;
                }
                const int held = t / 4 == grp ? pid_cur : pid_prev;
                for (int part = 0; part < PARTS; ++part, ++it) {
                    const int e = it % E;
                    int freed = 0;
                    if (lane == 0) freed = mbar_wait(&empty_bar[e], (((uint32_t)(it / E)) & 1u) ^ 1u, abort_ptr) ? 1 : 0;
                    if (!__shfl_sync(0xffffffffu, freed, 0)) { ok = false; break; }
                    if (lane == 0) mbar_expect_tx(&ready_bar[e], (uint32_t)Cfg::kEntry);
                    __syncwarp();
                    // K parts are halves of d, V parts halves of the positions
                    const int groups = is_v ? NCH : NCH / PARTS, pages = Cfg::kBoxes / groups;
                    const int c = lane % groups, pg = lane / groups;
                    const int dc = is_v ? c : part * groups + c, page = (is_v ? part * pages : 0) + pg;
                    int pid = __shfl_sync(0xffffffffu, held, (t % 4) * kPagesPerBlock + page % kPagesPerBlock);
                    if (lane < Cfg::kBoxes) {
                        if (pid < 0 || pid >= p.a.num_pages) { set_status(p.a.dev_status, MASSV_ERR_CAPACITY); pid = 0; }
                        tma_load_2d(smem + (size_t)e * Cfg::kEntry + c * (pages * kPageSize * 128) + pg * 2048, is_v ? &map_v : &map_k, dc * 64,
                                    (pid * p.a.Hkv + sg.head) * kPageSize, &ready_bar[e], policy);
                    }
                }
            }
        }
        if (lane == 0 && *abort_ptr) {
            for (int i = 0; i < 64; ++i) __nanosleep(2000);            // let copies in flight land
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
            int tau[2] = {0, 0}, segs[2] = {0, 0};   // blocks and segments so far, by tile
            auto entry_ready = [&](int i) { if (ok && !mbar_wait(&ready_bar[i % E], ((uint32_t)(i / E)) & 1u, abort_ptr)) ok = false; };
            // S = Q_x K^T over `d_part`'s share of d (the whole of it with one part)
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
            // O_x (+)= P V over `part`'s share of the positions
            auto pv = [&](int x, int buf, int i, int part, bool first) {
                const uint32_t v_lo = (((ring + (uint32_t)(i % E) * Cfg::kEntry) & 0x3FFFFu) >> 4) | ((uint32_t)(kVRegion >> 4) << 16);
                const uint32_t d_tmem = tmem_base + Cfg::kTmemO + (uint32_t)(x * D), a0 = tmem_base + (uint32_t)(buf * kPrefixBlock);
#pragma unroll
                for (int ks = 0; ks < kPrefixBlock / 16 / PARTS; ++ks) {
                    const uint32_t a = a0 + (uint32_t)((part * (kPrefixBlock / 16 / PARTS) + ks) * 8), bb = v_lo + (uint32_t)((ks * 2048) >> 4);
                    if (ks == 0 && part == 0 && first) umma_bf16_ts<false>(d_tmem, a, bb, idesc_pv);
                    else umma_bf16_ts<true>(d_tmem, a, bb, idesc_pv);
                }
            };
            for (int seg = 0; ok && next_segment(sg); ++seg) {
                const int n = sg.n;
                const bool two = sg.n_rows[1] > 0;
                if (!mbar_wait(&q_ready_bar, (uint32_t)seg & 1u, abort_ptr)) { ok = false; break; }
                if constexpr (NT == 2) {
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
                            if (x == 0 || two) {
                                if (ok && !mbar_wait(&p_full_bar[x], (uint32_t)(tau[x] + t) & 1u, abort_ptr)) ok = false;
                                if (ok && t == 0 && segs[x] > 0 && !mbar_wait(&o_free_bar[x], (uint32_t)(segs[x] - 1) & 1u, abort_ptr)) ok = false;
                                if (!ok) break;
                                tc_fence_after();
                                pv(x, x, iv, 0, t == 0);
                            }
                            if (x == (two ? 1 : 0)) umma_commit(&empty_bar[iv % E]);
                            if (x == 1 && !two) break;
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
                    tau[0] += n; segs[0] += 1;
                    if (two) { tau[1] += n; segs[1] += 1; }
                } else {
                    auto scores = [&](int t) {
                        const int buf = (tau[0] + t) & 1;             // its last P was read by a product issued before
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
                    for (int t = 0; t < n && ok; ++t) {
                        if (t + 1 < n) scores(t + 1);
                        const int at = tau[0] + t, buf = at & 1;
                        if (ok && !mbar_wait(&p_full_bar[buf], (uint32_t)(at >> 1) & 1u, abort_ptr)) ok = false;
                        if (ok && t == 0 && segs[0] > 0 && !mbar_wait(&o_free_bar[0], (uint32_t)(segs[0] - 1) & 1u, abort_ptr)) ok = false;
#pragma unroll
                        for (int part = 0; part < PARTS; ++part, ++it) {
                            entry_ready(it);
                            if (!ok) break;
                            tc_fence_after();
                            pv(0, buf, it, part, t == 0);
                            umma_commit(&empty_bar[it % E]);
                        }
                        if (!ok) break;
                        umma_commit(&pv_done_bar);
                        if (t == n - 1) umma_commit(&o_full_bar[0]);
                    }
                    tau[0] += n; segs[0] += 1;
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
        int tau = 0, segs = 0;
        while (ok && next_segment(sg)) {
            if (sg.n_rows[x] == 0) continue;
            float ref = -INFINITY, l_run = 0.f;
            for (int t = 0; t < sg.n && ok; ++t, ++tau) {
                const int buf = NT == 2 ? x : tau & 1;
                const uint32_t parity = (uint32_t)(NT == 2 ? tau : tau >> 1) & 1u;
                if (!mbar_wait_warp(&s_full_bar[buf], parity, abort_ptr)) { ok = false; break; }
                tc_fence_after();
                const uint32_t tmem_s = tmem_base + lane_base + (uint32_t)(buf * kPrefixBlock);
                uint32_t s[kPrefixBlock];
#pragma unroll
                for (int c = 0; c < kPrefixBlock; c += 32) tmem_ld_row32(tmem_s + (uint32_t)c, s + c);
                tmem_ld_wait(s);
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
                    // (two tiles: the scores stand behind the product before them, so O is up to date)
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
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&p_full_bar[buf]);
            }
            if (!ok || !mbar_wait_warp(&o_full_bar[x], (uint32_t)segs & 1u, abort_ptr)) { ok = false; break; }
            ++segs;
            tc_fence_after();
            // ---- the result: merged with the rest and written, or a piece
            const int blk = sg.blk0 + x * nb + row / G;
            const bool live = row < sg.n_rows[x] && p.skip[blk / p.a.R] > 0;
            if (sg.whole) {
                const size_t at = live ? (size_t)blk * p.a.Hq + sg.head * G + row % G : 0;
                const float lse1 = ref + log2f(l_run), lse2 = live ? p.tail_lse[at] * 1.4426950408889634f : 0.f, m = fmaxf(lse1, lse2);
                const float w1 = exp2f(lse1 - m), w2 = exp2f(lse2 - m), inv = 1.f / (w1 + w2), f1 = w1 * inv / l_run, f2 = w2 * inv;
#pragma unroll 1
                for (int c0 = 0; c0 < D; c0 += 32) {
                    uint32_t o[32];
                    tmem_ld_row32(tmem_o + (uint32_t)c0, o);
                    tmem_ld_wait(o);
                    if (live && MASSV_IN_BOUNDS(at, (size_t)p.a.B * p.a.R * p.a.Hq, p.a.dev_status)) {
                        float4* rest = reinterpret_cast<float4*>(p.tail_out + at * D + c0);
                        uint4* dst = reinterpret_cast<uint4*>(p.a.out + at * D + c0);
#pragma unroll
                        for (int k = 0; k < 32; k += 8) {
                            float4 u = rest[k / 4], v = rest[k / 4 + 1];
                            u.x = u.x * f2 + __uint_as_float(o[k]) * f1; u.y = u.y * f2 + __uint_as_float(o[k + 1]) * f1;
                            u.z = u.z * f2 + __uint_as_float(o[k + 2]) * f1; u.w = u.w * f2 + __uint_as_float(o[k + 3]) * f1;
                            v.x = v.x * f2 + __uint_as_float(o[k + 4]) * f1; v.y = v.y * f2 + __uint_as_float(o[k + 5]) * f1;
                            v.z = v.z * f2 + __uint_as_float(o[k + 6]) * f1; v.w = v.w * f2 + __uint_as_float(o[k + 7]) * f1;
                            dst[k / 8] = make_uint4(bf16x2(u.x, u.y), bf16x2(u.z, u.w), bf16x2(v.x, v.y), bf16x2(v.z, v.w));
                            if (p.a.out_f32) { rest[k / 4] = u; rest[k / 4 + 1] = v; }
                        }
                    }
                }
                if (live && p.a.lse) p.a.lse[at] = (m + log2f(w1 + w2)) * 0.6931471805599453f;
            } else {
                int slot = sg.slot;
                if (!MASSV_IN_BOUNDS(slot, 2 * kPrefixMaxCtas, p.a.dev_status)) slot = 0;
                // a piece: unit c4 * 128 + row holds four columns of a row
                float4* dst = reinterpret_cast<float4*>(p.part_o) + ((size_t)slot * p.slot_tiles + x) * (kTileRows * D / 4) + row;
#pragma unroll 1
                for (int c0 = 0; c0 < D; c0 += 32) {
                    uint32_t o[32];
                    tmem_ld_row32(tmem_o + (uint32_t)c0, o);
                    tmem_ld_wait(o);
#pragma unroll
                    for (int k = 0; k < 32; k += 4)
                        dst[((c0 + k) / 4) * kTileRows] = make_float4(__uint_as_float(o[k]), __uint_as_float(o[k + 1]), __uint_as_float(o[k + 2]), __uint_as_float(o[k + 3]));
                }
                reinterpret_cast<float2*>(p.part_ml)[((size_t)slot * p.slot_tiles + x) * kTileRows + row] = make_float2(ref, l_run);
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

// Merge of the pieces of a cut tile and the rest.  CTA (c, tile): the item that runs out of the range of the prefix kernel's CTA c;
// thread (row, chunk) has 32 columns of a row.  Pieces are added in order.
__global__ void __launch_bounds__(1024) attn_prefix_merge_kernel(const SharedAttnParams p, int tiles_per_item) {
    const int c = blockIdx.x, x = blockIdx.y, row = threadIdx.x, c0 = threadIdx.y * 32, D = p.a.d;
    const int G = p.a.Hq / p.a.Hkv, nb = kTileRows / G;
    pdl_wait();
    pdl_trigger();
    const int* cum = p.meta + 1;
    const int per_cta = p.meta[0], total = cum[p.n_groups];
    const long long begin = (long long)c * per_cta;
    if (begin >= total) return;
    const PrefixItem it = prefix_item(p, cum, (int)min((long long)total, begin + per_cta) - 1);
    const int c_last = (it.start + it.blocks - 1) / per_cta;
    if (it.start / per_cta != c || c_last == c) return;          // begun by an earlier CTA, or not cut
    const int4 gr = p.groups[it.g];
    const int done = (it.tile * tiles_per_item + x) * nb, n_rows = min(nb, gr.w - done) * G;
    const int blk = gr.z + done + row / G;
    const bool live = row < n_rows && p.skip[blk / p.a.R] > 0;
    const size_t at = live ? (size_t)blk * p.a.Hq + it.head * G + row % G : 0;
    const float lse2 = live ? p.tail_lse[at] * 1.4426950408889634f : 0.f;
    __syncthreads();                                             // every chunk has read the rest's sum: the merged one may go over it
    if (!live) return;
    auto slot_of = [&](int k) { return ((size_t)k * 2 + (it.start <= k * per_cta ? 0 : 1)) * p.slot_tiles + x; };
    const float2* ml = reinterpret_cast<const float2*>(p.part_ml) + row;
    float m = lse2;
    for (int k = c; k <= c_last; ++k) m = fmaxf(m, ml[slot_of(k) * kTileRows].x);
    const float w2 = exp2f(lse2 - m);
    float sum = w2, acc[32];
    const float4* rest = reinterpret_cast<const float4*>(p.tail_out + at * D + c0);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const float4 v = rest[k];
        acc[4 * k] = v.x * w2; acc[4 * k + 1] = v.y * w2; acc[4 * k + 2] = v.z * w2; acc[4 * k + 3] = v.w * w2;
    }
    for (int k = c; k <= c_last; ++k) {
        const size_t slot = slot_of(k);
        const float2 v = ml[slot * kTileRows];
        const float w = exp2f(v.x - m);
        sum += v.y * w;
        const float4* src = reinterpret_cast<const float4*>(p.part_o) + slot * (kTileRows * D / 4) + (c0 / 4) * kTileRows + row;
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const float4 o = src[q * kTileRows];
            acc[4 * q] += o.x * w; acc[4 * q + 1] += o.y * w; acc[4 * q + 2] += o.z * w; acc[4 * q + 3] += o.w * w;
        }
    }
    const float inv = 1.f / sum;
#pragma unroll
    for (int k = 0; k < 32; ++k) acc[k] *= inv;
    uint4* dst = reinterpret_cast<uint4*>(p.a.out + at * D + c0);
#pragma unroll
    for (int k = 0; k < 32; k += 8)
        dst[k / 8] = make_uint4(bf16x2(acc[k], acc[k + 1]), bf16x2(acc[k + 2], acc[k + 3]), bf16x2(acc[k + 4], acc[k + 5]), bf16x2(acc[k + 6], acc[k + 7]));
    if (p.a.out_f32) {
        float4* f = reinterpret_cast<float4*>(p.a.out_f32 + at * D + c0);
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] = make_float4(acc[4 * k], acc[4 * k + 1], acc[4 * k + 2], acc[4 * k + 3]);
    }
    if (p.a.lse && c0 == 0) p.a.lse[at] = (m + log2f(sum)) * 0.6931471805599453f;
}

template <int D>
cudaError_t launch_prefix(const SharedAttnParams& p, const CUtensorMap& mk, const CUtensorMap& mv, cudaStream_t stream) {
    using Cfg = PrefixCfg<D>;
    const int G = p.a.Hq / p.a.Hkv;
    CUtensorMap mq;
    if (!make_tensor_map_bf16_heads(&mq, p.a.q, (uint64_t)p.a.B * p.a.R, (uint64_t)p.a.Hq, D, (uint32_t)(kTileRows / G), (uint32_t)G)) return cudaErrorInvalidValue;
    cudaError_t e = cudaFuncSetAttribute(attn_prefix_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg::kSmem);
    if (e != cudaSuccess) return e;
    int ctas = device_sm_count();
    if (ctas > kPrefixMaxCtas) ctas = kPrefixMaxCtas;
    e = launch_pdl(attn_prefix_kernel<D>, dim3(ctas), dim3(Cfg::kThreads), (size_t)Cfg::kSmem, stream, mk, mv, mq, p);
    if (e != cudaSuccess) return e;
    return launch_pdl(attn_prefix_merge_kernel, dim3(ctas, p.slot_tiles), dim3(kTileRows, D / 32), 0, stream, p, Cfg::kTiles);
}

}  // namespace

int shared_attn_slot_tiles(int d, long rows) { return d == 256 || rows <= kTileRows ? 1 : 2; }

cudaError_t launch_shared_attn(const SharedAttnParams& p, const AttnParams& rest, cudaStream_t stream) {
    cudaError_t e = launch_pdl(attn_tail_kernel, dim3(p.a.B), dim3(128), 0, stream, p);
    if (e != cudaSuccess) return e;
    e = launch_verify_attn(rest, stream);                      // (counts its own launches)
    if (e != cudaSuccess) return e;
    CUtensorMap mk, mv;
    const uint64_t rows_total = (uint64_t)p.a.num_pages * p.a.Hkv * kPageSize;
    if (!make_tensor_map_bf16_2d(&mk, p.a.k_pages, rows_total, p.a.d, kPageSize) || !make_tensor_map_bf16_2d(&mv, p.a.v_pages, rows_total, p.a.d, kPageSize))
        return cudaErrorInvalidValue;
    switch (p.a.d) {
        case 64: e = launch_prefix<64>(p, mk, mv, stream); break;
        case 128: e = launch_prefix<128>(p, mk, mv, stream); break;
        case 256: e = launch_prefix<256>(p, mk, mv, stream); break;
        default: return cudaErrorInvalidValue;
    }
    if (e != cudaSuccess) return e;
    count_launches(3);
    return cudaGetLastError();
}

}  // namespace massv
