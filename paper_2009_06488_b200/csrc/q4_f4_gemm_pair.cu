// e2m1 product with microscales on CTA pairs (clusters of two, tcgen05.mma.cta_group::2 block_scale): dense or by
// experts' rows.
//
//   C[m][n] = f sum_g SA[m][g] SB[n][g] sum_{k in group g} A[m][k] Bt[n][k]
//
// The tensor core applies the scales, so a tile's whole depth is summed in tensor memory.  A tile is 256 rows x BN
// columns (128 rows and BN columns per CTA).
//
//   warp 0       TMA producer   per stage (256 depth values): the CTA's 128 rows of A and its half of the tile's rows of
//                               Bt, 128 bytes each, 128-byte swizzle; rows past the end of the segment are not loaded
//   warp 1       MMA issuer     (leader CTA) a stage's scales to tensor memory (two buffers), then four products
//   warps 2..7   scales         words of the CTA's 128 rows of A and of all the tile's rows of Bt, put in atoms
//   warps 8..15  epilogue       each thread one row and BN / 2 columns: times f, rounded, out through swizzled staging slices
//                               and TMA stores (whole 32-row groups of aligned rows) or by pieces
//
// Bound: the ring of stages and a tile's end.  A stage of a wide tile lasts about 720 clk where its four products take 512 (without
// the scales' loads 8192^3 takes 169 us; with four stages instead of five 210; L2 runs at a quarter of its rate), and the only
// wide accumulator that fits beside the scales is drained for some 3000 clk per tile.  8192^3 to bf16: by 16 195 to 206 us = 5.3 to 5.6
// PFLOP/s, by 32 183 to 186 us = 5.9 to 6.0 (four times the bf16 product's measured rate is 6.6); under the power
// cap 222 to 245.  Scales by TMA boxes: 290 us; two accumulators of 192 columns: as long as one of 256.
#include <cuda.h>

#include "q4_f4_tc.cuh"

namespace q4 {
namespace f4 {

constexpr int TMC = 128;                 // rows of A per CTA
constexpr int FEW = 32;                  // rows of the smaller box of A
constexpr int NTHREADS = 16 * 32;
constexpr int SLICE = 4096;              // staging slice of an epilogue warp: 32 rows x 128 bytes

template <int BN, bool BY16> struct Cfg {
    static constexpr int WORDS = kWords<BY16>;
    static constexpr int BSH = BN / 2;                         // rows of Bt staged per CTA
    static constexpr int CW = BN / 2;                          // columns of an epilogue warp
    static constexpr int BATOMS = (BN + 127) / 128;            // atoms of Bt's scales per word
    static constexpr int SCALES = WORDS * (1 + BATOMS) * ATOM;
    static constexpr int STAGE = (TMC + BSH) * ROWB + SCALES;
    static constexpr int STAGES = BN == 256 ? 5 : 6;
    static constexpr int PARTS = 1 + BATOMS, TEAMS = 6 / PARTS;      // warps that bring a stage's scales, and how many of these
    static constexpr int ACCS = BN == 256 ? 1 : 2;
    static constexpr int COL_SCALE = ACCS * BN;                // tensor memory: accumulators, then two buffers of scales
    static constexpr int SCALE_COLS = WORDS * (1 + BATOMS) * 4;
    static constexpr int OFF_SLICE = STAGES * STAGE;
    static constexpr int OFF_BAR = OFF_SLICE + 8 * SLICE;
    static constexpr int NBAR = 2 * STAGES + 2 * ACCS;
    static constexpr int OFF_MISC = OFF_BAR + NBAR * 8;
    static constexpr int SMEM = OFF_MISC + 16 + 1024;          // + slack to align the base
    static_assert(STAGES >= TEAMS && STAGE % 1024 == 0 && SMEM <= 232448 && COL_SCALE + 2 * SCALE_COLS <= 512, "shared or tensor memory");
};

struct PairParams {
    GemmParams g;
    int32_t tiles_m, tiles_n;
    int32_t c_vec;                   // rows of C begin on multiples of 16 bytes (and tmC is valid)
};

// A store whose lines leave L2 ahead of the operands', which other tiles read again.
__device__ __forceinline__ void tma_store_2d_first(const CUtensorMap* tm, uint32_t src, int x, int y, uint64_t policy)
{
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group.L2::cache_hint [%0, {%2, %3}], [%1], %4;"
                 ::"l"(tm), "r"(src), "r"(x), "r"(y), "l"(policy) : "memory");
}

// A slice (32 rows x 128 bytes, its 16-byte pieces swizzled by the row) to rows of C by pieces: `rows` of them, `cols`
// columns (any number) from dst on, pitch in elements.
template <typename U>
__device__ __forceinline__ void put_slice(uint32_t slice, U* dst, int64_t pitch, int rows, int cols, bool vec, int lane)
{
    constexpr int PER = 128 / (int)sizeof(U), PIECE = 16 / (int)sizeof(U);
    cols = min(cols, PER);
    if (vec) {
        // aligned rows: 16 bytes per lane, the last piece of a ragged row by values
        for (int i = lane; i < rows * 8; i += 32) {
            const int r = i >> 3, c = i & 7;
            const int have = cols - c * PIECE;
            if (have <= 0) continue;
            const uint4 v = lds128(slice + (uint32_t)(r * 128) + (uint32_t)(((c ^ r) & 7) << 4));
            U* const at = dst + r * pitch + c * PIECE;
            if (have >= PIECE) {
                *reinterpret_cast<uint4*>(at) = v;
            } else {
                const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int j = 0; j < PIECE; ++j)
                    if (j < have) at[j] = sizeof(U) == 4 ? (U)w[j & 3] : (U)(w[(j >> 1) & 3] >> (16 * (j & 1)));
            }
        }
        return;
    }
    // rows that begin anywhere: by values, a warp's 32 of a row together; those of eight rows are read ahead of their stores
    for (int c = lane; c < PER; c += 32) {
        const int b = c * (int)sizeof(U);
#pragma unroll 1
        for (int r0 = 0; r0 < rows; r0 += 8) {
            U v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int r = r0 + k;
                const uint32_t w = (uint32_t)lds32(slice + (uint32_t)(r * 128) + (uint32_t)((((b >> 4) ^ r) & 7) << 4) + (uint32_t)(b & 12));
                v[k] = sizeof(U) == 4 ? (U)w : (U)(w >> (8 * (b & 2)));
            }
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (c < cols && r0 + k < rows) dst[(r0 + k) * pitch + c] = v[k];
        }
    }
}

template <int BN, bool BY16>
__global__ void __launch_bounds__(NTHREADS, 1)
gemm_f4_pair_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmAfew,
                    const __grid_constant__ CUtensorMap tmB, const __grid_constant__ CUtensorMap tmC,
                    const PairParams p)
{
    using C = Cfg<BN, BY16>;
    constexpr int CW = C::CW;
    extern __shared__ uint8_t smem_raw[];
    // the same offset in both CTAs: dynamic shared memory starts at the same address
    const uint32_t sbase = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t bar0 = sbase + C::OFF_BAR;
    auto bar_full   = [&](uint32_t s) { return bar0 + 8u * s; };                             // used in the leader
    auto bar_empty  = [&](uint32_t s) { return bar0 + 8u * (C::STAGES + s); };
    auto bar_tfull  = [&](uint32_t a) { return bar0 + 8u * (2 * C::STAGES + a); };
    auto bar_tempty = [&](uint32_t a) { return bar0 + 8u * (2 * C::STAGES + C::ACCS + a); };  // used in the leader
    const uint32_t tmem_slot = sbase + C::OFF_MISC;
    const uint32_t abort_flag = sbase + C::OFF_MISC + 4;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const GemmParams& g = p.g;
    const uint32_t rank = cluster_ctarank() & 1u;
    const int cluster_id = (int)blockIdx.x / 2, nclusters = (int)gridDim.x / 2;
    const int nkb = (g.K + STAGE_K - 1) / STAGE_K;

    if (threadIdx.x == 0) {
        for (int s = 0; s < C::STAGES; ++s) {
            mbar_init(bar_full(s), 2 + 2 * C::PARTS);        // an announcement of copies and the scales' warps per CTA
            mbar_init(bar_empty(s), 1);      // the leader's commit
        }
        for (int a = 0; a < C::ACCS; ++a) {
            mbar_init(bar_tfull(a), 1);
            mbar_init(bar_tempty(a), 16);    // epilogue warps of both CTAs
        }
        sts32(abort_flag, 0);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async_smem();
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(tmem_slot), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    cluster_sync_all();              // barriers of both CTAs are initialised past this point
    tc_fence_after();
    const uint32_t tmem_base = (uint32_t)lds32(tmem_slot);
    // every role waits for the kernel before ahead of its first access to global memory and of its first bounded wait
    f8::wait_for_predecessor();

    Walk<256, BN> walk(p.g, p.tiles_m, p.tiles_n, lane);
    Tile t;
    if (warp == 0) {
        // ------------------------------------------------------------ TMA producer
        const uint32_t full_leader = map_to_cta(bar_full(0), 0);
        uint32_t st = 0, ph = 0;
        for (int tile = cluster_id; walk.get(tile, t) && !lds32(abort_flag); tile += nclusters) {
            const int arow = t.m0 + (int)rank * TMC;
            const int rows = clamp_to(t.m_end - arow, 0, TMC);
            const int few = (rows + FEW - 1) / FEW;
            const uint32_t bytes = (uint32_t)((rows > TMC - FEW ? TMC : few * FEW) + C::BSH) * ROWB;
            for (int b = 0; b < nkb; ++b) {
                const bool ok = mbar_wait_or_leave(bar_empty(st), ph ^ 1u, abort_flag, g.status);
                if (elect_one() && ok) {
                    const uint32_t full = full_leader + 8u * st;
                    mbar_expect_tx_cluster(full, bytes);
                    const uint32_t dst = sbase + st * C::STAGE;
                    if (rows > TMC - FEW) tma_load_2d_pair(dst, &tmA, b * ROWB, arow, full);
                    else
                        for (int i = 0; i < few; ++i)
                            tma_load_2d_pair(dst + i * FEW * ROWB, &tmAfew, b * ROWB, arow + i * FEW, full);
                    tma_load_2d_pair(dst + TMC * ROWB, &tmB, b * ROWB, (int)t.brow + C::BSH * (int)rank, full);
                }
                __syncwarp();
                if (++st == C::STAGES) { st = 0; ph ^= 1u; }
            }
        }
        settle(abort_flag);
    } else if (warp == 1) {
        // ------------------------------------------------------------ pair MMA issuer (leader)
        if (rank == 0) {
            const uint64_t desc0 = make_kmajor_sw128_desc(sbase), scales0 = scales_desc(sbase + (TMC + C::BSH) * ROWB);
            uint32_t st = 0, ph = 0, buf = 0, acc = 0, aph = 0;
            for (int tile = cluster_id; walk.get(tile, t) && !lds32(abort_flag); tile += nclusters) {
                mbar_wait(bar_tempty(acc), aph ^ 1u, abort_flag, g.status);
                tc_fence_after();
                for (int b = 0; b < nkb; ++b) {
                    mbar_wait_or_leave<true>(bar_full(st), ph, abort_flag, g.status);
                    tc_fence_after();
                    if (elect_one()) {
                        const uint64_t adesc = desc0 + (uint64_t)(st * (uint32_t)(C::STAGE >> 4)), bdesc = adesc + (TMC * ROWB >> 4);
                        const uint64_t sdesc = scales0 + (uint64_t)(st * (uint32_t)(C::STAGE >> 4));
                        const uint32_t sa = tmem_base + C::COL_SCALE + buf * C::SCALE_COLS, sb = sa + 4 * C::WORDS;
#pragma unroll
                        for (int i = 0; i < C::WORDS * (1 + C::BATOMS); ++i)
                            tc_copy_scales<2>(sa + 4 * i, sdesc + (uint64_t)(i * (ATOM >> 4)));
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const int w = BY16 ? k : k >> 1;
                            tc_mma_f4<BY16, 2>(tmem_base + acc * BN, adesc + 2 * k, bdesc + 2 * k, idesc<BY16>(256, BN, BY16 ? 0 : 2 * (k & 1)),
                                               sa + 4 * w, sb + 4 * C::BATOMS * w, b | k ? 1u : 0u);
                        }
                        tc_commit_pair(bar_empty(st), 3);
                        if (b == nkb - 1) tc_commit_pair(bar_tfull(acc), 3);
                    }
                    __syncwarp();
                    buf ^= 1u;
                    if (++st == C::STAGES) { st = 0; ph ^= 1u; }
                }
                if (++acc == C::ACCS) { acc = 0; aph ^= 1u; }
            }
            settle(abort_flag);
        }
    } else if (warp < 8) {
        // ------------------------------------------------------------ scales
        // of a team's warps one brings the words of A, one each those of 128 rows of Bt
        const int part = (warp - 2) % C::PARTS, team = (warp - 2) / C::PARTS;
        const uint32_t full_leader = map_to_cta(bar_full(0), 0);
        int tile = cluster_id, b = team;
        bool more = walk.get(tile, t);
        bring_scales<C::WORDS, BY16, C::STAGES, C::TEAMS>(team, g.K, abort_flag,
            [&](const uint32_t*& src, int64_t& ld, int& rows, int& word0) {
                while (more && b >= nkb) {
                    b -= nkb;
                    more = walk.get(tile += nclusters, t);
                }
                if (!more) return false;
                const int row0 = t.m0 + (int)rank * TMC;
                src = (part ? g.SB + t.brow + 128 * (part - 1) : g.SA + row0) + lane;
                ld = part ? g.ldsb : g.ldsa;
                rows = (part ? g.N - t.n0 - 128 * (part - 1) : t.m_end - row0) - lane;
                word0 = b * C::WORDS;
                b += C::TEAMS;
                return true;
            },
            [&](uint32_t it, const uint4 (&v)[C::WORDS]) {
                const uint32_t st = it % C::STAGES, ph = it / C::STAGES & 1u;
                mbar_wait(bar_empty(st), ph ^ 1u, abort_flag, g.status);
                const uint32_t dst = sbase + st * C::STAGE + (TMC + C::BSH) * ROWB + (uint32_t)lane * 16u;
#pragma unroll
                for (int w = 0; w < C::WORDS; ++w)
                    sts128(dst + (uint32_t)((part ? C::WORDS + w * C::BATOMS + part - 1 : w) * ATOM), v[w]);
                // The leader's products read this CTA's atoms: the proxy fence and, behind the meeting, a release of shared
                // memory to the cluster.  (A releasing arrival waits for the loads under way as well, 320 us for 8192^3; through
                // a warp of its own that has none, 410.  The fence costs nothing that can be measured.)
                fence_async_smem();
                __syncwarp();
                fence_release_smem_cluster();
                if (lane == 0) mbar_arrive_cluster_relaxed(full_leader + 8u * st);
            });
    } else {
        // ------------------------------------------------------------ epilogue
        const int lg = warp & 3, set = warp >= 12 ? 1 : 0;
        const uint32_t tempty_leader = map_to_cta(bar_tempty(0), 0);
        const uint32_t slice = sbase + C::OFF_SLICE + (uint32_t)((warp - 8) * SLICE);
        const uint32_t mine = slice + (uint32_t)(lane * 128), sw = (uint32_t)(lane & 7);
        const float fa = g.FA ? __ldg(g.FA) : 1.0f;
        uint64_t evict_first;
        asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(evict_first));
        uint32_t acc = 0, aph = 0;
        for (int tile = cluster_id; walk.get(tile, t) && !lds32(abort_flag); tile += nclusters) {
            const int row0 = t.m0 + (int)rank * TMC + lg * 32, c0 = t.n0 + set * CW;
            const int rows = t.m_end - row0;
            const bool live = rows > 0 && c0 < g.N;
            const float f = fa * (g.FB ? __ldg(g.FB + t.e) : 1.0f);
            mbar_wait(bar_tfull(acc), aph, abort_flag, g.status);
            tc_fence_after();
            const uint32_t ta = tmem_base + ((uint32_t)(lg * 32) << 16) + acc * BN + (uint32_t)(set * CW);
            const uint32_t tempty = tempty_leader + 8u * acc;
            if (++acc == C::ACCS) { acc = 0; aph ^= 1u; }
            auto release = [&]() {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster_relaxed(tempty);
            };
            if (!live) {
                release();
                continue;
            }
            // a slice is in shared memory: out with it
            auto flush = [&](int nc, int per) {
                if (p.c_vec && rows >= 32 && (nc + per <= g.N || (int64_t)g.N * (128 / per) % 16 == 0)) {
                    fence_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        tma_store_2d_first(&tmC, slice, nc, row0, evict_first);
                        bulk_commit();
                    }
                } else {
                    __syncwarp();
                    const int64_t at = (int64_t)row0 * g.ldc + nc;
                    if (g.c_type == Q4_F32)
                        put_slice(slice, static_cast<uint32_t*>(g.C) + at, g.ldc, min(rows, 32), g.N - nc, p.c_vec, lane);
                    else
                        put_slice(slice, static_cast<uint16_t*>(g.C) + at, g.ldc, min(rows, 32), g.N - nc, p.c_vec, lane);
                    __syncwarp();
                }
            };
            auto reuse = [&]() {                            // the slice's last store has read it
                if (lane == 0) bulk_wait_read();
                __syncwarp();
            };
            if (g.c_type == Q4_F32) {
#pragma unroll 1
                for (int q = 0; q < CW / 32; ++q) {
                    uint32_t r[32];
                    tc_ld32(ta + (uint32_t)(32 * q), r);
                    tc_wait_ld32(r);
                    if (q == CW / 32 - 1) release();
                    if (c0 + 32 * q >= g.N) continue;
                    reuse();
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        sts128(mine + (((uint32_t)j ^ sw) << 4),
                               make_uint4(__float_as_uint(__uint_as_float(r[4 * j]) * f), __float_as_uint(__uint_as_float(r[4 * j + 1]) * f),
                                          __float_as_uint(__uint_as_float(r[4 * j + 2]) * f), __float_as_uint(__uint_as_float(r[4 * j + 3]) * f)));
                    flush(c0 + 32 * q, 32);
                }
            } else {
                // all columns to registers, rounded: the accumulator is free before anything is written
                uint32_t h[CW / 2];
#pragma unroll
                for (int q = 0; q < CW / 32; ++q) {
                    uint32_t r[32];
                    tc_ld32(ta + (uint32_t)(32 * q), r);
                    tc_wait_ld32(r);
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const float x = __uint_as_float(r[2 * j]) * f, y = __uint_as_float(r[2 * j + 1]) * f;
                        h[16 * q + j] = g.c_type == Q4_BF16 ? f8::pack2(x, y, (const __nv_bfloat16*)nullptr)
                                                            : f8::pack2(x, y, (const __half*)nullptr);
                    }
                }
                release();
#pragma unroll
                for (int q = 0; q < CW / 64; ++q) {
                    if (c0 + 64 * q >= g.N) break;
                    reuse();
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        sts128(mine + (((uint32_t)j ^ sw) << 4),
                               make_uint4(h[32 * q + 4 * j], h[32 * q + 4 * j + 1], h[32 * q + 4 * j + 2], h[32 * q + 4 * j + 3]));
                    flush(c0 + 64 * q, 64);
                }
            }
        }
        if (lane == 0) bulk_wait_read();       // my stores have read their slice; their writes complete with the grid
    }
    __syncwarp();
    tc_fence_before();
    cluster_sync_all();      // no CTA leaves or frees tensor memory while the other may still use it
    tc_fence_after();
    if (warp == 1)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
}

template <int BN, bool BY16>
static q4_status launch_pair(const PairParams& p, const CUtensorMap& a, const CUtensorMap& few, const CUtensorMap& b,
                             const CUtensorMap& c, int64_t clusters, cudaStream_t st)
{
    using Cf = Cfg<BN, BY16>;
    auto kernel = gemm_f4_pair_kernel<BN, BY16>;
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
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(clusters * 2));
    cfg.blockDim = dim3(NTHREADS);
    cfg.dynamicSmemBytes = Cf::SMEM;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, a, few, b, c, p);
    count_launch();
    return e == cudaSuccess ? Q4_OK : Q4_ERR_CUDA;
}

}  // namespace f4

using namespace f4;

bool gemm_f4_pair_supported(const f4::GemmParams& g)
{
    // A's rows of a tile may pass M by up to a tile; the maps count rows in 32 bits
    return (uintptr_t)g.A % 16 == 0 && (uintptr_t)g.Bt % 16 == 0 && g.lda % 16 == 0 && g.ldb % 16 == 0 &&
           g.M < INT32_MAX - 512 && (int64_t)g.N * (g.E ? g.E : 1) < INT32_MAX - 512;
}

q4_status launch_gemm_f4_pair(const f4::GemmParams& g, bool by16, cudaStream_t st)
{
    PairParams p{};
    p.g = g;
    p.tiles_m = (g.M + 255) / 256;
    const int pairs = f8_pairs_of_device();
    const int64_t n256 = ((int64_t)g.N + 255) / 256, n128 = ((int64_t)g.N + 127) / 128;
    const int64_t tm = p.tiles_m + (g.E ? (g.E < g.M ? g.E : g.M) : 0);          // an expert's last row tile is its own
    // Tile width: clocks of the busiest pair, from measured ones per stage (720 wide, 490 narrow) and tile.  1024 x 4096 x 4096
    // (64 wide tiles, one round; 128 narrow, two) 11.6 against 12.4 us, 512 x 4096 x 4096 10.6 against 8.7.
    const int64_t stages = ((int64_t)g.K + STAGE_K - 1) / STAGE_K;
    const int64_t t_wide = (tm * n256 + pairs - 1) / pairs * (stages * 720 + 3000);
    const int64_t t_narrow = (tm * n128 + pairs - 1) / pairs * (stages * 490 + 2500);
    const bool wide = g.N > 128 && t_wide <= t_narrow;
    p.tiles_n = (int)(wide ? n256 : n128);
    const size_t es = f8::type_size(g.c_type);
    p.c_vec = (uintptr_t)g.C % 16 == 0 && g.ldc * es % 16 == 0;
    const int kbytes = (g.K + 1) / 2;
    CUtensorMap a, few, b, c{};
    if (!make_byte_map(&a, g.A, g.lda, g.M, kbytes, TMC) || !make_byte_map(&few, g.A, g.lda, g.M, kbytes, FEW) ||
        !make_byte_map(&b, g.Bt, g.ldb, (int)((int64_t)g.N * (g.E ? g.E : 1)), kbytes, wide ? 128 : 64)) return Q4_ERR_CUDA;
    if (p.c_vec && !f8::make_out_map(&c, g.C, g.c_type, g.ldc, g.M, g.N)) return Q4_ERR_CUDA;
    const int64_t tiles = tm * p.tiles_n, clusters = tiles < pairs ? tiles : pairs;
    if (wide) return by16 ? launch_pair<256, true>(p, a, few, b, c, clusters, st) : launch_pair<256, false>(p, a, few, b, c, clusters, st);
    return by16 ? launch_pair<128, true>(p, a, few, b, c, clusters, st) : launch_pair<128, false>(p, a, few, b, c, clusters, st);
}

}  // namespace q4
