// e4m3 product with block scales on CTA pairs (clusters of two, tcgen05.mma.cta_group::2): dense, by experts'
// rows, or by experts' depth.
//
//   C[m][n] = sum over blocks b of 128 depth values of  SA[b][m] * SB(n, b) * P_b[m][n],   P_b = sum_k a b
//
// The scales change with the depth, so the tensor core may only sum inside a block: P_b comes to tensor
// memory, and 8 warps per CTA take it from there into binary32 registers, acc = fma(P_b, SA * SB, acc), while
// the next blocks are multiplied.  A tile is 256 rows x BN = 128 * HALVES columns (128 rows per CTA).
//
//   warp 0       TMA producer    per block: the CTA's 128 rows of A and its half of the tile's rows of Bt, 128 bytes
//                                each, 128-byte swizzle; rows past the end of the segment are not loaded
//   warps 1, 2   MMA issuers     (leader CTA) four 32-deep steps per block and 128 columns
//   warp 3       places          of the tiles, found ahead for the accumulators
//   warps 4..11  accumulators    each thread one row and BN / 2 columns; then scaled sums out through swizzled
//                                staging slices and TMA stores (whole 32-row groups of aligned rows) or aligned 16-byte pieces cut
//                                from them (ragged groups, rows that begin anywhere)
//
// Tensor memory holds four slots of 128 columns.  With HALVES = 2 each column half has two of them and its own
// four accumulating warps, so a half's drain (and the two hand-offs around it) has three quarters of the
// two blocks' tensor time; one slot of 256 columns per block would leave it half.
//
// Bound: the drain.  A block of a wide tile is 512 clk of tensor time; the accumulators need about 750 for it
// (eight loads of 16 columns, each followed by its multiply-adds, 460 clk for the two warps of a scheduler; the
// wait, the scales and the release the rest).  What was tried beside it: sixteen accumulating warps of 64 columns
// (issue slots bind: 4096^3 72 to 78 us), 32-column loads (they slow the products beside them: 87 us), a second
// buffer (the loads of one warp do not overlap its arithmetic: no change), waiting for the next block before the
// last multiply-adds (70 us), a warp that multiplies the scales for all (76 us).  In long runs the power cap binds:
// 8192^3 430 to 460 us = 2.4 to 2.6 PFLOP/s in a short region, 527 us = 2.09 PFLOP/s at about 1.4 GHz in a long one.
//
// With SPLIT the cluster is 2 * splits CTAs that share one tile's depth; their partial tiles are added in
// order through distributed shared memory (problems of few tiles).
#include <cuda.h>

#include "q4_f8.cuh"
#include "q4_tc_ptx.cuh"

namespace q4 {

bool make_byte_map(CUtensorMap* tm, const uint8_t* base, int64_t ld, int rows, int kbytes, int box_rows);

namespace f8 {

constexpr int TMC = 128;                 // rows of A per CTA
constexpr int ROWB = 128;                // bytes (= depth values) per row per stage: one block of scales
constexpr int FEW = 32;                  // rows of the smaller box of A
constexpr int NTHREADS = 12 * 32;
// Registers: the block is launched with 384 x 168 = 64512; warps 0..3 give back to 56 each, the accumulators
// take 224 (128 x 56 + 256 x 224 = 64512).
constexpr int REGS_ISSUE = 56, REGS_ACC = 224;
constexpr int TI_RING = 3;               // tiles whose places are staged for the accumulators
constexpr int SLICE = 4096;              // staging slice of an accumulator warp: 32 rows x 128 bytes

template <int HALVES, bool BROWS> struct Cfg {
    static constexpr int BN = 128 * HALVES;
    static constexpr int BSH = BN / 2;                         // rows of Bt staged per CTA
    static constexpr int CW = BN / 2;                          // columns of an accumulator warp
    static constexpr int STAGE = (TMC + BSH) * ROWB;
    static constexpr int STAGES = HALVES == 2 ? (BROWS ? 4 : 5) : 6;
    static constexpr int OFF_SLICE = STAGES * STAGE;
    static constexpr int OFF_SB = OFF_SLICE + 8 * 2 * SLICE;   // [set][buffer][4 blocks][CW] scales of Bt's rows
    static constexpr int OFF_TI = OFF_SB + (BROWS ? 2 * 2 * 4 * CW * 4 : 0);    // places of tiles
    static constexpr int OFF_BAR = OFF_TI + TI_RING * 32;
    static constexpr int NBAR = 2 * STAGES + 8 + 2 * TI_RING + 2;
    static constexpr int OFF_MISC = OFF_BAR + NBAR * 8;
    static constexpr int SMEM = OFF_MISC + 16 + 1024;          // + slack to align the base
    static_assert(STAGE % 1024 == 0 && SMEM <= 232448, "shared memory");
    static_assert(128 * (BN + 4) * 4 <= OFF_SLICE || HALVES == 2, "split partials fit the ring");
};

// D = f32, A = B = e4m3, K-major, M = 256 (pair), N = 128.
constexpr uint32_t kIdesc = (1u << 4) | ((uint32_t)(128 >> 3) << 17) | ((uint32_t)(256 >> 4) << 24);

__device__ __forceinline__ void tc_mma_f8_pair(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(kIdesc), "r"(accumulate) : "memory");
}
// Waits for the thread's tensor-memory loads; the loaded registers pass through it, so that nothing that
// uses them can be moved above it.
__device__ __forceinline__ void tc_wait_ld16(uint32_t (&r)[16])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                   "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
                 :: "memory");
}
__device__ __forceinline__ unsigned long long pack_f2(uint32_t lo, uint32_t hi)
{
    unsigned long long v;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "r"(lo), "r"(hi));
    return v;
}
__device__ __forceinline__ void unpack_f2(unsigned long long v, uint32_t& lo, uint32_t& hi)
{
    asm("mov.b64 {%0, %1}, %2;" : "=r"(lo), "=r"(hi) : "l"(v));
}
__device__ __forceinline__ void fma_f2(unsigned long long& acc, unsigned long long a, unsigned long long b)
{
    asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(acc) : "l"(a), "l"(b));
}
__device__ __forceinline__ unsigned long long mul_f2(unsigned long long a, unsigned long long b)
{
    unsigned long long v;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(a), "l"(b));
    return v;
}
__device__ __forceinline__ uint4 lds128_cluster(uint32_t a)
{
    uint4 v;
    asm volatile("ld.shared::cluster.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}

__device__ __forceinline__ void prefetch_map(const CUtensorMap* m)
{
    asm volatile("prefetch.tensormap [%0];" ::"l"(m) : "memory");
}

// A load that stays where it is written (the compiler would move a plain one down to its use, a round of four
// blocks later, and expose its latency); 0 where `in` is false.
__device__ __forceinline__ float load_ahead(const float* at, bool in)
{
    float v;
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %2, 0;\n\tmov.f32 %0, 0f00000000;\n\t"
                 "@p ld.global.nc.f32 %0, [%1];\n\t}" : "=f"(v) : "l"(at), "r"((int)in) : "memory");
    return v;
}

struct PairParams {
    GemmF8Params g;
    int32_t tiles_m, tiles_n;        // kDense, kExpertDepth: of one product
    int32_t splits;
    int32_t c_vec;                   // rows of C begin on multiples of 16 bytes (and tmC is valid)
};

struct Tile {
    int m0, m_end;                   // first row of the pair's tile and end of its segment (rows of A)
    int n0;                          // first column
    int64_t arow, brow;              // rows of A and Bt in their maps
    int64_t crow;                    // C row of m0
    int64_t sbrow;                   // row of SB (by block)
    int k0, nkb;                     // first depth value, blocks
};

__device__ __forceinline__ int clamp_to(int v, int lo, int hi) { return min(max(v, lo), hi); }

// The walk over the tiles.  Called by whole warps: an expert's segment is found 32 experts at a time.
template <int BN>
struct Walk {
    const PairParams& p;
    int lane;
    int e0 = 0, cum = 0, lo = 0, hi = 0, incl = 0;
    __device__ Walk(const PairParams& p_, int lane_) : p(p_), lane(lane_)
    {
        if (p.g.mode == kExpertRows) load();
    }
    __device__ void load()
    {
        const int e = e0 + lane;
        lo = hi = 0;
        if (e < p.g.E) {
            lo = clamp_to(p.g.starts[e], 0, p.g.M);
            hi = clamp_to(p.g.starts[e + 1], lo, p.g.M);
        }
        incl = (hi - lo + 255) / 256 * p.tiles_n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int u = __shfl_up_sync(0xFFFFFFFFu, incl, o);
            if (lane >= o) incl += u;
        }
    }
    __device__ bool get(int t, Tile& o)
    {
        const GemmF8Params& g = p.g;
        o.k0 = 0;
        o.nkb = (g.K + ROWB - 1) / ROWB;
        if (g.mode == kExpertRows) {
            int total = __shfl_sync(0xFFFFFFFFu, incl, 31);
            while (t >= cum + total) {
                if (e0 + 32 >= g.E) return false;
                cum += total;
                e0 += 32;
                load();
                total = __shfl_sync(0xFFFFFFFFu, incl, 31);
            }
            const int i = __popc(__ballot_sync(0xFFFFFFFFu, t - cum >= incl));
            const int before = i ? __shfl_sync(0xFFFFFFFFu, incl, i - 1) : 0;
            const int s = __shfl_sync(0xFFFFFFFFu, lo, i), end = __shfl_sync(0xFFFFFFFFu, hi, i);
            const int tm = (end - s + 255) / 256;
            const int local = t - cum - before, n = local / tm;        // row tiles fastest: they share the weights
            o.m0 = s + (local - n * tm) * 256;
            o.m_end = end;
            o.n0 = n * BN;
            o.arow = o.crow = o.m0;
            o.brow = (int64_t)(e0 + i) * g.N + o.n0;
            o.sbrow = (e0 + i) * blocks_of(g.N) + o.n0 / BLK;
            return true;
        }
        const int per = p.tiles_m * p.tiles_n;
        int e = 0, local = t;
        if (g.mode == kExpertDepth) {
            e = t / per;
            if (e >= g.E) return false;
            local = t - e * per;
            // block boundaries: starts are rounded down, the depth's own end stays (an empty segment there is empty too)
            const int a = clamp_to(g.starts[e], 0, g.K), b = clamp_to(g.starts[e + 1], a, g.K);
            o.k0 = a / ROWB * ROWB;
            o.nkb = a == b ? 0 : b == g.K ? (b - o.k0 + ROWB - 1) / ROWB : (b / ROWB * ROWB - o.k0) / ROWB;
        } else if (t >= per) {
            return false;
        }
        // bands of eight row tiles: the tiles in flight at a time share rows of both operands
        const int band = local / (8 * p.tiles_n), r = local - band * 8 * p.tiles_n;
        const int h = min(8, p.tiles_m - band * 8), n = r / h;
        o.m0 = (band * 8 + r - n * h) * 256;
        o.m_end = g.M;
        o.n0 = n * BN;
        o.arow = o.m0;
        o.brow = o.n0;
        o.crow = (int64_t)e * g.M + o.m0;
        o.sbrow = o.n0 / BLK;
        return true;
    }
};

template <int HALVES, bool BROWS, bool SPLIT>
__global__ void __launch_bounds__(NTHREADS, 1)
gemm_f8_pair_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmAfew,
                    const __grid_constant__ CUtensorMap tmB, const __grid_constant__ CUtensorMap tmC,
                    const PairParams p)
{
    using C = Cfg<HALVES, BROWS>;
    constexpr int BN = C::BN, CW = C::CW;
    extern __shared__ uint8_t smem_raw[];
    // the same offset in every CTA: dynamic shared memory starts at the same address
    const uint32_t sbase = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t bar0 = sbase + C::OFF_BAR;
    auto bar_full   = [&](int s) { return bar0 + 8u * (uint32_t)s; };                        // used in the leader
    auto bar_empty  = [&](int s) { return bar0 + 8u * (uint32_t)(C::STAGES + s); };
    auto bar_tfull  = [&](int a) { return bar0 + 8u * (uint32_t)(2 * C::STAGES + a); };
    auto bar_tempty = [&](int a) { return bar0 + 8u * (uint32_t)(2 * C::STAGES + 4 + a); };  // used in the leader
    auto bar_ifull  = [&](uint32_t i) { return bar0 + 8u * (2 * C::STAGES + 8 + i); };           // a tile's place is staged
    auto bar_iempty = [&](uint32_t i) { return bar0 + 8u * (2 * C::STAGES + 8 + TI_RING + i); };
    auto bar_set    = [&](int i) { return bar0 + 8u * (uint32_t)(2 * C::STAGES + 8 + 2 * TI_RING + i); };   // a set's warps meet (BROWS)
    const uint32_t tmem_slot = sbase + C::OFF_MISC;
    const uint32_t abort_flag = sbase + C::OFF_MISC + 4;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const GemmF8Params& g = p.g;
    const uint32_t cta = cluster_ctarank();
    const uint32_t rank = cta & 1u, leader = cta & ~1u;
    const int splits = SPLIT ? p.splits : 1, split = SPLIT ? (int)(cta >> 1) : 0;
    const int cluster_id = (int)blockIdx.x / (2 * splits), nclusters = (int)gridDim.x / (2 * splits);

    if (threadIdx.x == 0) {
        for (int s = 0; s < C::STAGES; ++s) {
            mbar_init(bar_full(s), 2);       // one announcement per CTA's producer
            mbar_init(bar_empty(s), HALVES);  // the leader's commits, one per issuer that reads the stage
        }
        for (int a = 0; a < 4; ++a) {
            mbar_init(bar_tfull(a), 1);
            mbar_init(bar_tempty(a), HALVES == 2 ? 8 : 16);   // accumulator warps of both CTAs that read the slot
        }
        for (uint32_t i = 0; i < TI_RING; ++i) {
            mbar_init(bar_ifull(i), 1);
            mbar_init(bar_iempty(i), 8);     // accumulator warps
        }
        mbar_init(bar_set(0), 4);
        mbar_init(bar_set(1), 4);
        sts32(abort_flag, 0);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async_smem();
    }
    if (warp == 0 && elect_one()) {
        prefetch_map(&tmA);
        prefetch_map(&tmAfew);
        prefetch_map(&tmB);
        if (p.c_vec) prefetch_map(&tmC);
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(tmem_slot), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    cluster_sync_all();              // barriers of all CTAs are initialised past this point
    tc_fence_after();
    const uint32_t tmem_base = (uint32_t)lds32(tmem_slot);
    // Every warp of the roles below waits for the kernel before ahead of its first access to global memory and of its first
    // bounded wait: what another warp does only behind it may take as long as that kernel runs.  What needs neither comes
    // first and overlaps its end, the places of a dense product's first tile with it.
    const bool dense = g.mode == kDense;

    // the share of a tile's depth blocks that this pair sums
    auto share = [&](Tile& t) {
        if (SPLIT) {
            const int lo = (int)((int64_t)t.nkb * split / splits), hi = (int)((int64_t)t.nkb * (split + 1) / splits);
            t.k0 += lo * ROWB;
            t.nkb = hi - lo;
        }
    };

    Tile t;
    if (warp == 0) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS_ISSUE));
        // ------------------------------------------------------------ TMA producer
        if (!dense) wait_for_predecessor();
        Walk<BN> walk(p, lane);
        const uint32_t full_leader = map_to_cta(bar_full(0), leader);
        uint32_t st = 0, ph = 0;
        Tile next;
        bool more = walk.get(cluster_id, next);
        if (dense) wait_for_predecessor();
        for (int tile = cluster_id; more;) {
            t = next;
            share(t);
            const int rows = clamp_to(t.m_end - t.m0 - (int)rank * TMC, 0, TMC);
            const int arow = (int)t.arow + (int)rank * TMC;
            const int halves = HALVES == 2 && g.N - t.n0 > 128 ? 2 : 1;
            const int few = (rows + FEW - 1) / FEW;
            const uint32_t bytes = (uint32_t)((rows > TMC - FEW ? TMC : few * FEW) + halves * 64) * ROWB;
            for (int b = 0; b < t.nkb; ++b) {
                mbar_wait(bar_empty(st), ph ^ 1u, abort_flag, g.status);
                if (elect_one()) {
                    const uint32_t full = full_leader + 8u * st;
                    mbar_expect_tx_cluster(full, bytes);
                    const uint32_t dst = sbase + st * C::STAGE;
                    const int x = t.k0 + b * ROWB;
                    if (rows > TMC - FEW) tma_load_2d_pair(dst, &tmA, x, arow, full);
                    else
                        for (int i = 0; i < few; ++i)
                            tma_load_2d_pair(dst + i * FEW * ROWB, &tmAfew, x, arow + i * FEW, full);
                    for (int h = 0; h < halves; ++h)
                        tma_load_2d_pair(dst + (TMC + 64 * h) * ROWB, &tmB, x, (int)t.brow + 128 * h + 64 * (int)rank, full);
                }
                __syncwarp();
                if (++st == C::STAGES) { st = 0; ph ^= 1u; }
            }
            more = walk.get(tile += nclusters, next) && !lds32(abort_flag);
        }
        __syncwarp();
        cluster_sync_all();
        if (SPLIT) cluster_sync_all();
    } else if (warp < 3) {
        // ------------------------------------------------------------ pair MMA issuers (leader)
        // Each block's product has a slot of its own, so its order does not matter.  One warp's waits and commits
        // for a block take longer than its multiplication: two warps share them, by column half, or by blocks
        // in turn where there is one half.
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS_ISSUE));
        if (rank == 0) {
            const int who = warp - 1;
            if (!dense) wait_for_predecessor();
            Walk<BN> walk(p, lane);
            const uint16_t both = (uint16_t)(3u << leader);
            const uint64_t desc0 = make_kmajor_sw128_desc(sbase);
            const uint64_t bstep = (uint64_t)((TMC + (HALVES == 2 ? 64 * who : 0)) * ROWB >> 4);
            uint32_t st = 0, ph = 0, u = 0;
            Tile next;
            bool more = walk.get(cluster_id, next);
            if (dense) wait_for_predecessor();
            for (int tile = cluster_id; more;) {
                t = next;
                share(t);
                tile += nclusters;
                if (t.nkb == 0) more = walk.get(tile, next);
                const bool empty = HALVES == 2 && who == 1 && g.N - t.n0 <= 128;     // no such half
                for (int b = 0; b < t.nkb; ++b) {
                    if (b == 1 || t.nkb == 1) more = walk.get(tile, next);     // while the first block is multiplied
                    if (HALVES == 2 || (int)(u & 1u) == who) {
                        mbar_wait(bar_full(st), ph, abort_flag, g.status);
                        tc_fence_after();
                        if (!empty) {
                            const int slot = HALVES == 2 ? who * 2 + (int)(u & 1u) : (int)(u & 3u);
                            const uint32_t sph = (HALVES == 2 ? u >> 1 : u >> 2) & 1u;
                            mbar_wait(bar_tempty(slot), sph ^ 1u, abort_flag, g.status);
                            tc_fence_after();
                            const uint64_t adesc = desc0 + (uint64_t)(st * (uint32_t)(C::STAGE >> 4));
                            if (elect_one()) {
#pragma unroll
                                for (int i = 0; i < 4; ++i)
                                    tc_mma_f8_pair(tmem_base + (uint32_t)(slot * 128), adesc + (uint64_t)(2 * i),
                                                   adesc + bstep + (uint64_t)(2 * i), i ? 1u : 0u);
                                tc_commit_pair(bar_tfull(slot), both);
                            }
                        }
                        if (elect_one()) tc_commit_pair(bar_empty(st), both);
                        __syncwarp();
                    }
                    if (HALVES == 1 || !empty) ++u;
                    if (++st == C::STAGES) { st = 0; ph ^= 1u; }
                }
                if (lds32(abort_flag)) break;
            }
        }
        __syncwarp();
        tc_fence_before();
        cluster_sync_all();      // no CTA leaves or frees tensor memory while another may still use it
        if (SPLIT) cluster_sync_all();
        tc_fence_after();
        if (warp == 1)
            asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
    } else if (warp == 3) {
        // ------------------------------------------------------------ places of tiles, for the accumulators
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS_ISSUE));
        if (!dense) wait_for_predecessor();
        Walk<BN> walk(p, lane);
        uint32_t ti = 0, ph = 0;
        for (int tile = cluster_id;; tile += nclusters) {
            const bool more = walk.get(tile, t);
            if (more) share(t);
            mbar_wait_suspend(bar_iempty(ti), ph ^ 1u, abort_flag, g.status);
            const bool last = !more || lds32(abort_flag);
            if (lane == 0) {
                const uint32_t at = sbase + C::OFF_TI + ti * 32u;
                sts128(at, make_uint4((uint32_t)t.m0, (uint32_t)t.m_end, (uint32_t)t.n0, last ? 0xFFFFFFFFu : (uint32_t)t.nkb));
                sts128(at + 16u, make_uint4((uint32_t)(t.k0 / ROWB), (uint32_t)t.sbrow, (uint32_t)t.crow, (uint32_t)(t.crow >> 32)));
                mbar_arrive(bar_ifull(ti));
            }
            __syncwarp();
            if (last) break;
            if (dense && tile == cluster_id) wait_for_predecessor();
            if (++ti == TI_RING) { ti = 0; ph ^= 1u; }
        }
        __syncwarp();
        cluster_sync_all();
        if (SPLIT) cluster_sync_all();
    } else {
        // ------------------------------------------------------------ accumulators
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS_ACC));
        wait_for_predecessor();
        const int lg = warp & 3, set = warp >= 8 ? 1 : 0;
        const uint32_t tempty_leader = map_to_cta(bar_tempty(0), leader);
        const uint32_t slices = sbase + C::OFF_SLICE + (uint32_t)((warp - 4) * 2 * SLICE);
        const uint32_t sb_s = sbase + C::OFF_SB + (uint32_t)(set * 2 * 4 * CW * 4);
        const int st_id = lg * 32 + lane;                 // thread of the set
        uint32_t used = 0, ti = 0, tph = 0;
        uint32_t met = 0;
        auto meet = [&]() {                                // the set's four warps; bounded like every wait
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_set(set));
            mbar_wait(bar_set(set), met, abort_flag, g.status);
            met ^= 1u;
        };
        // the tile whose scales are loaded: this one, or from its last round on the next
        int f_c0 = 0, f_rows = 0, f_nkb = -1, nkb = -1;  // first column, valid rows from my warp's first, blocks (-1: no tile)
        const float *sa_at = nullptr, *sb_at = nullptr;
        float sa[4], sb[4];
        // scales of blocks b0 .. b0 + 3, loaded a round of four blocks ahead
        auto fetch = [&](int b0) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool in = b0 + i < f_nkb;
                sa[i] = load_ahead(sa_at + (b0 + i) * g.ldsa, in && f_rows > lane);
                if (!BROWS) {
                    sb[i] = load_ahead(sb_at + b0 + i, in && f_c0 < g.N);
                } else if (i < 4 * CW / 128) {
                    const int el = i * 128 + st_id, kb = el / CW, n = f_c0 + el % CW;
                    sb[i] = load_ahead(sb_at + (b0 + kb) * g.ldsb + n, b0 + kb < f_nkb && n < g.N);
                }
            }
        };
        // the next tile's place and its first scales
        auto next = [&](uint32_t i, uint32_t ph) {
            mbar_wait(bar_ifull(i), ph, abort_flag, g.status);
            const uint4 x = lds128(sbase + C::OFF_TI + i * 32u), y = lds128(sbase + C::OFF_TI + i * 32u + 16u);
            const int m0 = (int)x.x + (int)rank * TMC + lg * 32;
            f_nkb = lds32(abort_flag) ? -1 : (int)x.w;
            if (f_nkb < 0) return;
            f_c0 = (int)x.z + set * CW;
            f_rows = (int)x.y - m0;
            if (HALVES == 2 && set == 1 && g.N - (int)x.z <= 128) f_nkb = 0;     // nothing is multiplied in my half
            sa_at = g.SA + (int64_t)y.x * g.ldsa + m0 + lane;
            sb_at = g.SB + (BROWS ? (int64_t)y.x * g.ldsb : ((int64_t)y.y + (HALVES == 2 ? set : 0)) * g.ldsb + y.x);
            fetch(0);
        };
        next(0, 0);
        while ((nkb = f_nkb) >= 0) {
            const bool live = f_rows > 0 && f_c0 < g.N;
            const uint32_t ti_next = ti + 1 == TI_RING ? 0 : ti + 1, tph_next = ti + 1 == TI_RING ? tph ^ 1u : tph;
            unsigned long long acc[CW / 2];
#pragma unroll
            for (int i = 0; i < CW / 2; ++i) acc[i] = 0;
#pragma unroll 1
            for (int b0 = 0; b0 < nkb; b0 += 4) {
                float s[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) s[i] = BROWS ? sa[i] : sa[i] * sb[i];
                const uint32_t sb_buf = sb_s + (uint32_t)(((b0 >> 2) & 1) * 4 * CW * 4);
                if (BROWS) {
                    // two buffers: a warp that writes one has passed the barrier behind which all read the other
#pragma unroll
                    for (int i = 0; i < 4 * CW / 128; ++i) sts32(sb_buf + 4u * (uint32_t)(i * 128 + st_id), __float_as_int(sb[i]));
                    meet();
                }
                if (b0 + 4 < nkb) fetch(b0 + 4);
                else next(ti_next, tph_next);
                const int n = min(4, nkb - b0);
#pragma unroll 1
                for (int i = 0; i < n; ++i) {
                    const uint32_t u = used++;
                    const int slot = HALVES == 2 ? set * 2 + (int)(u & 1u) : (int)(u & 3u);
                    mbar_wait(bar_tfull(slot), (HALVES == 2 ? u >> 1 : u >> 2) & 1u, abort_flag, g.status);
                    tc_fence_after();
                    const uint32_t tempty = tempty_leader + 8u * (uint32_t)slot;
                    if (live) {
                        const uint32_t ta = tmem_base + ((uint32_t)(lg * 32) << 16) +
                                            (uint32_t)(slot * 128 + (HALVES == 2 ? 0 : set * CW));
                        const uint32_t sbits = __float_as_uint(s[0]);
                        const unsigned long long ss = pack_f2(sbits, sbits);
#pragma unroll
                        for (int c = 0; c < CW / 16; ++c) {
                            uint32_t r[16];
                            tc_ld16(ta + (uint32_t)(16 * c), r);
                            tc_wait_ld16(r);
                            if (c + 1 == CW / 16) {
                                // my loads of the slot are complete: it may be overwritten
                                tc_fence_before();
                                __syncwarp();
                                if (lane == 0) mbar_arrive_cluster_relaxed(tempty);
                            }
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                if (BROWS) {
                                    const uint4 q = lds128(sb_buf + 4u * (uint32_t)(i * CW + 16 * c + 4 * j));
                                    fma_f2(acc[8 * c + 2 * j], mul_f2(pack_f2(r[4 * j], r[4 * j + 1]), pack_f2(q.x, q.y)), ss);
                                    fma_f2(acc[8 * c + 2 * j + 1], mul_f2(pack_f2(r[4 * j + 2], r[4 * j + 3]), pack_f2(q.z, q.w)), ss);
                                } else {
                                    fma_f2(acc[8 * c + 2 * j], pack_f2(r[4 * j], r[4 * j + 1]), ss);
                                    fma_f2(acc[8 * c + 2 * j + 1], pack_f2(r[4 * j + 2], r[4 * j + 3]), ss);
                                }
                            }
                        }
                    } else {
                        __syncwarp();
                        if (lane == 0) mbar_arrive_cluster_relaxed(tempty);
                    }
                    s[0] = s[1]; s[1] = s[2]; s[2] = s[3];
                }
            }
            if (BROWS && nkb > 0) meet();                 // buffers free for the next tile

            if (SPLIT) {
                // partial tile [128 rows][BN + 4] over the ring, which nothing reads or fills any more: this pair's
                // blocks are all multiplied
                const uint32_t part = sbase + (uint32_t)(((lg * 32 + lane) * (BN + 4) + set * CW) * 4);
#pragma unroll
                for (int i = 0; i < CW / 4; ++i) {
                    uint4 v;
                    unpack_f2(acc[2 * i], v.x, v.y);
                    unpack_f2(acc[2 * i + 1], v.z, v.w);
                    sts128(part + 16u * (uint32_t)i, v);
                }
            }
            if (nkb == 0) next(ti_next, tph_next);
            const uint4 x = lds128(sbase + C::OFF_TI + ti * 32u), y = lds128(sbase + C::OFF_TI + ti * 32u + 16u);
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_iempty(ti));
            ti = ti_next;
            tph = tph_next;
            if (!SPLIT && live) {
                const int c0 = (int)x.z + set * CW, rows = (int)x.y - ((int)x.x + (int)rank * TMC + lg * 32);
                const int64_t crow = (int64_t)((uint64_t)y.w << 32 | y.z) + (int)rank * TMC + lg * 32;     // C row of my warp's first
                const int es = g.c_type == Q4_F32 ? 4 : 2, per = 128 / es;      // columns per slice
                // slices q0 .. q1 - 1 to memory
                auto flush = [&](int q0, int q1) {
                    fence_async_smem();
                    __syncwarp();
                    int q = q0;
                    q1 = min(q1, CW / per);
                    // a store clips rows and columns at the matrix's end, columns in pieces of 16 bytes only
                    for (; p.c_vec && rows >= 32 && q < q1; ++q) {
                        const int nc = c0 + q * per;
                        if (nc >= g.N || (nc + per > g.N && g.N * es % 16 != 0)) break;
                        if (lane == 0) {
                            tma_store_2d(&tmC, slices + (uint32_t)((q & 1) * SLICE), nc, (int)crow);
                            bulk_commit();
                        }
                    }
                    const int nc = c0 + q * per, bytes = min((q1 - q) * 128, (g.N - nc) * es);
                    if (bytes <= 0) return;
                    // the rest in aligned pieces of 16 bytes, each cut from two of the slices', ...
                    uint8_t* const dst = static_cast<uint8_t*>(g.C) + (crow * g.ldc + nc) * es;
                    const int64_t pitch = g.ldc * es;
                    const int lg_pieces = q1 - q > 1 ? 4 : 3, n = min(rows, 32);
                    auto piece = [&](int r, int c) {
                        return slices + (uint32_t)(((q + (c >> 3)) & 1) * SLICE + r * 128) + (uint32_t)(((c ^ r) & 7) << 4);
                    };
                    // (four at a time: loads, then stores; every address lies in the warp's two slices)
                    const int total = n << lg_pieces, head0 = (int)(-(intptr_t)dst & 15), skew = (int)(pitch & 15);
#pragma unroll 1
                    for (int i0 = lane; i0 < total; i0 += 128) {
                        uint4 x[4], y[4];
#pragma unroll
                        for (int u = 0; u < 4; ++u) {
                            const int i = i0 + 32 * u, r = i >> lg_pieces & 31, c = i & ((1 << lg_pieces) - 1);
                            x[u] = lds128(piece(r, c));
                            y[u] = lds128(piece(r, c + 1));
                        }
#pragma unroll
                        for (int u = 0; u < 4; ++u) {
                            const int i = i0 + 32 * u, r = i >> lg_pieces, c = i & ((1 << lg_pieces) - 1);
                            const int head = (head0 - r * skew) & 15, off = head + 16 * c;
                            if (i < total && off + 16 <= bytes)
                                *reinterpret_cast<uint4*>(dst + r * pitch + off) = f8::cut16(x[u], y[u], head);
                        }
                    }
                    // ... and what is left at either end by values, a row's by eight lanes
                    const int ends = bytes & 15 ? 30 : head0 | skew ? 16 : 0;
#pragma unroll 1
                    for (int k = (lane & 7) * es; k < ends; k += 8 * es) {
#pragma unroll 1
                        for (int r0 = lane >> 3; r0 < n; r0 += 16) {
                            uint32_t v[4];
                            int off[4];
#pragma unroll
                            for (int u = 0; u < 4; ++u) {
                                const int r = r0 + 4 * u, head = min((head0 - r * skew) & 15, bytes), tail = (bytes - head) & 15;
                                off[u] = k < head ? k : bytes - tail + k - head;
                                if (r >= n || k >= head + tail) off[u] = -1;
                                const uint32_t from = piece(r & 31, max(off[u], 0) >> 4) + (uint32_t)(off[u] & 15);
                                v[u] = (uint32_t)lds32(from & ~3u) >> (8 * (from & 2u));
                            }
#pragma unroll
                            for (int u = 0; u < 4; ++u) {
                                uint8_t* const at = dst + (r0 + 4 * u) * pitch + off[u];
                                if (off[u] < 0) continue;
                                if (es == 4) *reinterpret_cast<uint32_t*>(at) = v[u];
                                else *reinterpret_cast<uint16_t*>(at) = (uint16_t)v[u];
                            }
                        }
                    }
                    __syncwarp();
                };
                const uint32_t mine = slices + (uint32_t)(lane * 128), sw = (uint32_t)(lane & 7);
                if (g.c_type == Q4_F32) {
                    // the first two slices together, then one at a time as the older one has been read (a slice
                    // that goes out without a bulk store is the warp's last, or all of them do)
#pragma unroll
                    for (int q0 = 0; q0 < CW / 32; q0 += q0 ? 1 : 2) {
                        if (c0 + q0 * 32 < g.N) {
                            if (lane == 0) {
                                if (q0) bulk_wait_read_but_one();
                                else bulk_wait_read();                 // the previous tile's
                            }
                            __syncwarp();
#pragma unroll
                            for (int j = 0; j < (q0 ? 8 : 16); ++j) {
                                uint4 v;
                                unpack_f2(acc[16 * q0 + 2 * j], v.x, v.y);
                                unpack_f2(acc[16 * q0 + 2 * j + 1], v.z, v.w);
                                sts128(mine + (uint32_t)(((q0 + (j >> 3)) & 1) * SLICE) + ((((uint32_t)j & 7u) ^ sw) << 4), v);
                            }
                            flush(q0, q0 ? q0 + 1 : 2);
                        }
                    }
                } else {
                    if (lane == 0) bulk_wait_read();
                    __syncwarp();
#pragma unroll
                    for (int j = 0; j < CW / 8; ++j) {
                        uint32_t w[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            uint32_t lo, hi;
                            unpack_f2(acc[4 * j + k], lo, hi);
                            const float x = __uint_as_float(lo), y = __uint_as_float(hi);
                            w[k] = g.c_type == Q4_BF16 ? pack2(x, y, (const __nv_bfloat16*)nullptr)
                                                       : pack2(x, y, (const __half*)nullptr);
                        }
                        sts128(mine + (uint32_t)((j >> 3) * SLICE) + ((((uint32_t)j & 7u) ^ sw) << 4),
                               make_uint4(w[0], w[1], w[2], w[3]));
                    }
                    flush(0, 2);
                }
            }
        }
        if (lane == 0) bulk_wait_read();       // my TMA stores have read their slices; their writes complete with the grid
        __syncwarp();
        tc_fence_before();
        cluster_sync_all();      // every partial tile is written; my tensor-memory loads are done
        if (SPLIT) {
            // one tile per cluster: CTA `split` of a rank adds its 128 / splits rows of all partial tiles, in order
            Walk<BN> walk(p, lane);
            if (walk.get(cluster_id, t)) {
                // eight rows of a warp at a time (all of them for two pairs or more): their loads are under way together
                const int col = t.n0 + lane * 4, have = min(4, g.N - col), end = (split + 1) * TMC / splits;
#pragma unroll 1
                for (int r0 = split * TMC / splits + warp - 4; r0 < end; r0 += 64) {
                    float v[8][4] = {};
#pragma unroll 1
                    for (int i = 0, s = split; i < splits; ++i, s = s + 1 == splits ? 0 : s + 1) {     // not all from one CTA at a time
                        const uint32_t part = map_to_cta(sbase, (uint32_t)s * 2 + rank) + (uint32_t)(lane * 16);
                        uint4 q[8];
#pragma unroll
                        for (int u = 0; u < 8; ++u) {
                            q[u] = make_uint4(0, 0, 0, 0);
                            if (r0 + 8 * u < end) q[u] = lds128_cluster(part + (uint32_t)((r0 + 8 * u) * (BN + 4) * 4));
                        }
#pragma unroll
                        for (int u = 0; u < 8; ++u) {
                            v[u][0] += __uint_as_float(q[u].x);
                            v[u][1] += __uint_as_float(q[u].y);
                            v[u][2] += __uint_as_float(q[u].z);
                            v[u][3] += __uint_as_float(q[u].w);
                        }
                    }
#pragma unroll
                    for (int u = 0; u < 8; ++u) {
                        const int r = r0 + 8 * u, row = (int)rank * TMC + r;
                        if (r >= end || t.m0 + row >= t.m_end || have <= 0) continue;
                        const int64_t at = (t.crow + row) * g.ldc + col;
                        if (g.c_type == Q4_F32) {
                            float* dst = static_cast<float*>(g.C) + at;
                            if (p.c_vec && have == 4) *reinterpret_cast<float4*>(dst) = make_float4(v[u][0], v[u][1], v[u][2], v[u][3]);
                            else
#pragma unroll
                                for (int j = 0; j < 4; ++j) if (j < have) dst[j] = v[u][j];
                        } else {
                            const bool bf = g.c_type == Q4_BF16;
                            const uint32_t w0 = bf ? pack2(v[u][0], v[u][1], (const __nv_bfloat16*)nullptr) : pack2(v[u][0], v[u][1], (const __half*)nullptr);
                            const uint32_t w1 = bf ? pack2(v[u][2], v[u][3], (const __nv_bfloat16*)nullptr) : pack2(v[u][2], v[u][3], (const __half*)nullptr);
                            uint16_t* dst = static_cast<uint16_t*>(g.C) + at;
                            if (p.c_vec && have == 4) {
                                *reinterpret_cast<uint2*>(dst) = make_uint2(w0, w1);
                            } else {
#pragma unroll
                                for (int j = 0; j < 4; ++j) if (j < have) dst[j] = (uint16_t)((j < 2 ? w0 : w1) >> (16 * (j & 1)));
                            }
                        }
                    }
                }
            }
            cluster_sync_all();      // the partial tiles have been read
        }
    }
}

// C [rows x cols], box = 128 bytes x 32 rows, read from a 128-byte-swizzled staging slice.
static bool make_out_map(CUtensorMap* tm, void* base, int type, int64_t ldc, int64_t rows, int cols)
{
    using Fn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                            const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                            CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static Fn fn = nullptr;
    if (!fn) {
        void* sym = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &sym, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess) return false;
        fn = reinterpret_cast<Fn>(sym);
    }
    const cuuint64_t es = type_size(type);
    cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    cuuint64_t strides[1] = {(cuuint64_t)ldc * es};
    cuuint32_t box[2] = {(cuuint32_t)(128 / es), 32};
    cuuint32_t estr[2] = {1, 1};
    const CUtensorMapDataType dt = type == Q4_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                 : type == Q4_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    return fn(tm, dt, 2, base, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int HALVES, bool BROWS, bool SPLIT>
static q4_status launch_pair(const PairParams& p, const CUtensorMap& a, const CUtensorMap& few, const CUtensorMap& b,
                             const CUtensorMap& c, int64_t clusters, cudaStream_t st)
{
    using Cf = Cfg<HALVES, BROWS>;
    auto kernel = gemm_f8_pair_kernel<HALVES, BROWS, SPLIT>;
    static bool ready[64] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return Q4_ERR_CUDA;
    if (!ready[dev]) {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Cf::SMEM) != cudaSuccess)
            return Q4_ERR_CUDA;
        ready[dev] = true;
    }
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)(2 * p.splits);
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(clusters * 2 * p.splits));
    cfg.blockDim = dim3(NTHREADS);
    cfg.dynamicSmemBytes = Cf::SMEM;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, a, few, b, c, p);
    count_launch();
    return e == cudaSuccess ? Q4_OK : Q4_ERR_CUDA;
}

// Clusters of `splits` pairs of the split kernel that run at once on the current device (splits 2..4).
static int clusters_of_device(int splits)
{
    static int per_dev[64][5] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
    int& n = per_dev[dev][splits];
    if (!n) {
        using Cf = Cfg<1, false>;
        auto kernel = gemm_f8_pair_kernel<1, false, true>;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = (unsigned)(2 * splits);
        attr[0].val.clusterDim.y = 1;
        attr[0].val.clusterDim.z = 1;
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3((unsigned)(2 * splits));
        cfg.blockDim = dim3(NTHREADS);
        cfg.dynamicSmemBytes = Cf::SMEM;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Cf::SMEM) != cudaSuccess ||
            cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess || n < 1) {
            cudaGetLastError();
            n = -1;
        }
    }
    return n;
}

}  // namespace f8

using namespace f8;

int f8_pairs_of_device()
{
    static int per_dev[64] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 74;
    if (!per_dev[dev]) {
        int n = 0;
        if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 2) n = 148;
        per_dev[dev] = n / 2;
    }
    return per_dev[dev];
}

bool gemm_f8_pair_supported(const GemmF8Params& g)
{
    // A's rows of a tile may pass M by up to a tile; the maps count rows in 32 bits
    return (uintptr_t)g.A % 16 == 0 && (uintptr_t)g.Bt % 16 == 0 && g.lda % 16 == 0 && g.ldb % 16 == 0 &&
           g.M < INT32_MAX - 512 && (int64_t)g.N * (g.mode == kExpertRows ? g.E : 1) < INT32_MAX - 512;
}

q4_status launch_gemm_f8_pair(const GemmF8Params& g, cudaStream_t st)
{
    PairParams p{};
    p.g = g;
    p.tiles_m = (g.M + 255) / 256;
    const int64_t nkb = blocks_of(g.K);
    const int pairs = f8_pairs_of_device();
    const int64_t products = g.mode == kExpertDepth ? g.E : 1;
    const int64_t n256 = ((int64_t)g.N + 255) / 256, n128 = ((int64_t)g.N + 127) / 128;
    // row tiles: an expert's last one is its own
    const int64_t tm = g.mode == kExpertRows ? p.tiles_m + (g.E < g.M ? g.E : g.M) : p.tiles_m * products;
    // Tile width: clocks of the busiest pair, from measured ones per block (780 wide, 480 narrow) and tile (2500).
    // 2048^3 (64 wide tiles, one round; 128 narrow, two) 13.0 against 13.9 us, 1024 x 4096 x 4096 19.4 against 21.8,
    // 4096^3 64 against 71; 512 x 2304 x 2304 takes narrow tiles, all in one round either way.
    const int64_t per = g.mode == kExpertDepth ? (nkb + g.E - 1) / g.E : nkb;
    const int64_t t_wide = (tm * n256 + pairs - 1) / pairs * (per * 780 + 2500);
    const int64_t t_narrow = (tm * n128 + pairs - 1) / pairs * (per * 480 + 2500);
    const bool wide = g.N > 128 && t_wide <= t_narrow;
    // Depth split of narrow tiles, again by measured clocks: 445 per block, 740 with scales by row, 1700 for the exchange and 90
    // for each pair that takes part in it; only while all clusters run at once (a cluster lies within a GPC, so 33 of four CTAs,
    // 22 of six and 15 of eight fit where 74 pairs do).  Whole, in two, three and four parts: 200 x 250 x 1024 7.0, 7.2, 6.8, 6.7
    // us, with scales by row 8.2, 7.7, 7.3, 7.0; 500 x 500 x 2048 7.9, 7.8, 7.5, 7.7; 1000 x 500 x 1024 6.1, 7.2, 8.0, -; 2304 x
    // 256 x 4097 by row 18.2, 14.0, 12.5, -; 100 x 4096 x 4096 (32 tiles) 11.5, 12.3, -, -.
    int splits = 1;
    if (!wide && g.mode != kExpertRows) {
        const int64_t block = g.b_rows ? 740 : 445;
        int64_t best = per * block;
        for (int k = 2; k <= 4; ++k) {
            const int64_t clk = (per + k - 1) / k * block + 1700 + 90 * tm * n128 * k;
            if (clk >= best || tm * n128 > clusters_of_device(k)) continue;
            best = clk;
            splits = k;
        }
    }
    p.splits = splits;
    p.tiles_n = (int)(wide ? n256 : n128);
    const size_t es = type_size(g.c_type);
    p.c_vec = (uintptr_t)g.C % 16 == 0 && g.ldc * es % 16 == 0;
    const int64_t crows = g.mode == kExpertDepth ? (int64_t)g.E * g.M : g.M;
    CUtensorMap a, few, b, c{};
    if (!make_byte_map(&a, g.A, g.lda, g.M, g.K, TMC) || !make_byte_map(&few, g.A, g.lda, g.M, g.K, FEW) ||
        !make_byte_map(&b, g.Bt, g.ldb, (int)(g.mode == kExpertRows ? (int64_t)g.E * g.N : g.N), g.K, 64)) return Q4_ERR_CUDA;
    if (p.c_vec && !make_out_map(&c, g.C, g.c_type, g.ldc, crows, g.N)) return Q4_ERR_CUDA;
    const int64_t tiles = tm * p.tiles_n;
    const int64_t clusters = splits > 1 || tiles < pairs ? tiles : pairs;
    if (wide) return g.b_rows ? launch_pair<2, true, false>(p, a, few, b, c, clusters, st)
                              : launch_pair<2, false, false>(p, a, few, b, c, clusters, st);
    if (splits > 1) return g.b_rows ? launch_pair<1, true, true>(p, a, few, b, c, clusters, st)
                                    : launch_pair<1, false, true>(p, a, few, b, c, clusters, st);
    return g.b_rows ? launch_pair<1, true, false>(p, a, few, b, c, clusters, st)
                    : launch_pair<1, false, false>(p, a, few, b, c, clusters, st);
}

}  // namespace q4
