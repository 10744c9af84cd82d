// e2m1 product with microscales for few rows of A (tokens being decoded): the weights' 128 rows are the instruction's rows
// and NB rows of A its columns, so that the weights' stream from HBM is what the kernel waits for.
//
//   C[m][n] = f sum_g SA[m][g] SB[n][g] sum_{k in group g} A[m][k] Bt[n][k]
//
//   warp 0       TMA producer   stages of 256 depth values: 128 rows of Bt, NB rows of A (128-byte swizzle)
//   warp 1       MMA issuer     a stage's scales to tensor memory (two buffers), then four products (tcgen05, one CTA)
//   warps 2..7   scales         teams of two: the words of the rows of Bt and of A, put in atoms
//   warps 8..11  epilogue       a thread per column of C, its NB values times f, rounded, to memory
//
// One persistent CTA per SM walks the tiles; with SPLIT a cluster of CTAs shares one tile's depth and adds its partial
// tiles through distributed shared memory, in order (a product of few tiles).
// Bound: HBM, behind the grid's start and ends.  A product of 128 rows takes about 118 clk for 64 depth values up to NB = 64 and 128
// at 128, 39 bytes of weights per clk and SM, where HBM brings 23.  Sixteen tokens of eight, 64 experts by 16 whose weights change
// from call to call: 2048 x 2048 23.3 us = 5.2 TB/s, 2048 x 1024 14.4 us = 4.2; one token through 4096 x 4096, by 16: 5.6 us.
#include <cuda.h>

#include "q4_f4_tc.cuh"

namespace q4 {
namespace f4 {

constexpr int FEW_THREADS = 12 * 32;
constexpr int WR = 128;                  // rows of Bt of a tile
constexpr int MAX_SPLITS = 8;            // parts of the depth

template <int NB, bool BY16> struct FewCfg {
    static constexpr int WORDS = kWords<BY16>;
    static constexpr int ATOMS = 2 * WORDS * ATOM;             // of Bt's rows, then of A's
    static constexpr int STAGE = (WR + NB) * ROWB + ATOMS;
    static constexpr int STAGES = NB <= 32 ? 8 : NB == 64 ? 6 : 5;
    static constexpr int TEAMS = 3;
    static constexpr int COLS = NB <= 64 ? 256 : 512;
    static constexpr int COL_SCALE = 2 * NB;                   // tensor memory: two accumulators, two buffers of scales
    static constexpr int OFF_BAR = STAGES * STAGE;
    static constexpr int OFF_MISC = OFF_BAR + (2 * STAGES + 4) * 8;
    static constexpr int SMEM = OFF_MISC + 16 + 1024;
    static_assert(NB * WR * 4 <= OFF_BAR && STAGE % 1024 == 0 && STAGES >= TEAMS && SMEM <= 232448 && COL_SCALE + 2 * 8 * WORDS <= COLS, "shared or tensor memory");
};

struct FewParams {
    GemmParams g;
    int32_t tiles_m, tiles_n, splits;
    int32_t c_vec;                   // four values of C at a time are aligned
};

__device__ __forceinline__ float4 lds128_cluster(uint32_t a)
{
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a) : "memory");
    return v;
}

template <int NB, bool BY16, bool SPLIT>
__global__ void __launch_bounds__(FEW_THREADS, 1)
gemm_f4_few_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const FewParams p)
{
    using C = FewCfg<NB, BY16>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t sbase = (smem_u32(smem_raw) + 1023u) & ~1023u;         // (alike in all CTAs of a cluster)
    const uint32_t bar0 = sbase + C::OFF_BAR;
    auto bar_full   = [&](uint32_t s) { return bar0 + 8u * s; };
    auto bar_empty  = [&](uint32_t s) { return bar0 + 8u * (C::STAGES + s); };
    auto bar_tfull  = [&](uint32_t a) { return bar0 + 8u * (2 * C::STAGES + a); };
    auto bar_tempty = [&](uint32_t a) { return bar0 + 8u * (2 * C::STAGES + 2 + a); };
    const uint32_t tmem_slot = sbase + C::OFF_MISC, abort_flag = tmem_slot + 4;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const GemmParams& g = p.g;
    const int split = SPLIT ? (int)cluster_ctarank() : 0, splits = SPLIT ? p.splits : 1;
    const int first = (int)blockIdx.x / splits, step = (int)gridDim.x / splits;
    const int blocks = (g.K + STAGE_K - 1) / STAGE_K;
    const int k_lo = (int)((int64_t)blocks * split / splits), nkb = (int)((int64_t)blocks * (split + 1) / splits) - k_lo;

    if (threadIdx.x == 0) {
        for (int s = 0; s < C::STAGES; ++s) {
            mbar_init(bar_full(s), 3);       // the copies' announcement, the two scales' warps
            mbar_init(bar_empty(s), 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(bar_tfull(a), 1);
            mbar_init(bar_tempty(a), 4);
        }
        sts32(abort_flag, 0);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async_smem();
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tmem_slot), "r"((uint32_t)C::COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = (uint32_t)lds32(tmem_slot);
    f8::wait_for_predecessor();

    Walk<NB, WR> walk(g, p.tiles_m, p.tiles_n, lane);
    Tile t;
    if (warp == 0) {
        // ------------------------------------------------------------ TMA producer
        uint32_t st = 0, ph = 0;
        for (int tile = first; walk.get(tile, t) && !lds32(abort_flag); tile += step)
            for (int b = 0; b < nkb; ++b) {
                const bool ok = mbar_wait_or_leave(bar_empty(st), ph ^ 1u, abort_flag, g.status);
                if (elect_one() && ok) {
                    const uint32_t dst = sbase + st * C::STAGE;
                    mbar_expect_tx(bar_full(st), (uint32_t)((WR + NB) * ROWB));
                    tma_load_2d(dst, &tmB, (k_lo + b) * ROWB, (int)t.brow, bar_full(st));
                    tma_load_2d(dst + WR * ROWB, &tmA, (k_lo + b) * ROWB, t.m0, bar_full(st));
                }
                __syncwarp();
                if (++st == C::STAGES) { st = 0; ph ^= 1u; }
            }
        settle(abort_flag);
    } else if (warp == 1) {
        // ------------------------------------------------------------ MMA issuer
        const uint64_t desc0 = make_kmajor_sw128_desc(sbase), scales0 = scales_desc(sbase + (WR + NB) * ROWB);
        uint32_t st = 0, ph = 0, buf = 0, acc = 0, aph = 0;
        for (int tile = first; walk.get(tile, t) && !lds32(abort_flag); tile += step) {
            mbar_wait(bar_tempty(acc), aph ^ 1u, abort_flag, g.status);
            for (int b = 0; b < nkb; ++b) {
                mbar_wait_or_leave(bar_full(st), ph, abort_flag, g.status);
                tc_fence_after();
                if (elect_one()) {
                    const uint64_t adesc = desc0 + (uint64_t)(st * (uint32_t)(C::STAGE >> 4)), bdesc = adesc + (WR * ROWB >> 4);
                    const uint64_t sdesc = scales0 + (uint64_t)(st * (uint32_t)(C::STAGE >> 4));
                    const uint32_t sa = tmem_base + C::COL_SCALE + buf * (8 * C::WORDS), sb = sa + 4 * C::WORDS;
#pragma unroll
                    for (int i = 0; i < 2 * C::WORDS; ++i) tc_copy_scales<1>(sa + 4 * i, sdesc + (uint64_t)(i * (ATOM >> 4)));
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int w = BY16 ? k : k >> 1;
                        tc_mma_f4<BY16, 1>(tmem_base + acc * NB, adesc + 2 * k, bdesc + 2 * k, idesc<BY16>(WR, NB, BY16 ? 0 : 2 * (k & 1)),
                                           sa + 4 * w, sb + 4 * w, b | k ? 1u : 0u);
                    }
                    tc_commit(bar_empty(st));
                    if (b == nkb - 1) tc_commit(bar_tfull(acc));
                }
                __syncwarp();
                buf ^= 1u;
                if (++st == C::STAGES) { st = 0; ph ^= 1u; }
            }
            aph ^= acc;
            acc ^= 1u;
        }
        settle(abort_flag);
    } else if (warp < 8) {
        // ------------------------------------------------------------ scales
        const int part = warp & 1, team = (warp - 2) >> 1;     // 0: Bt's rows, 1: A's
        int tile = first, b = team;
        bool more = walk.get(tile, t);
        bring_scales<C::WORDS, BY16, C::STAGES, C::TEAMS>(team, g.K, abort_flag,
            [&](const uint32_t*& src, int64_t& ld, int& rows, int& word0) {
                while (more && b >= nkb) {
                    b -= nkb;
                    more = walk.get(tile += step, t);
                }
                if (!more) return false;
                src = (part ? g.SA + t.m0 : g.SB + t.brow) + lane;
                ld = part ? g.ldsa : g.ldsb;
                rows = (part ? min(t.m_end - t.m0, NB) : g.N - t.n0) - lane;
                word0 = (k_lo + b) * C::WORDS;
                b += C::TEAMS;
                return true;
            },
            [&](uint32_t it, const uint4 (&v)[C::WORDS]) {
                const uint32_t st = it % C::STAGES, ph = it / C::STAGES & 1u;
                mbar_wait(bar_empty(st), ph ^ 1u, abort_flag, g.status);
                const uint32_t dst = sbase + st * C::STAGE + (WR + NB) * ROWB + (uint32_t)(part * C::WORDS * ATOM + lane * 16);
#pragma unroll
                for (int w = 0; w < C::WORDS; ++w) sts128(dst + (uint32_t)(w * ATOM), v[w]);
                fence_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar_full(st));
            });
    } else {
        // ------------------------------------------------------------ epilogue
        const int h = warp - 8;
        const float fa = g.FA ? __ldg(g.FA) : 1.0f;
        uint32_t acc = 0, aph = 0;
        for (int tile = first; walk.get(tile, t) && !lds32(abort_flag); tile += step) {
            const int n = t.n0 + 32 * h + lane, rows = min(NB, t.m_end - t.m0);
            const float f = fa * (g.FB ? __ldg(g.FB + t.e) : 1.0f);
            mbar_wait_suspend(bar_tfull(acc), aph, abort_flag, g.status);
            tc_fence_after();
            const uint32_t ta = tmem_base + ((uint32_t)(h * 32) << 16) + acc * NB;
#pragma unroll 1
            for (int j0 = 0; j0 < NB && j0 < rows; j0 += 16) {
                uint32_t r[16];
                tc_ld16(ta + (uint32_t)j0, r);
                tc_wait_ld16(r);
                const int64_t at = (int64_t)(t.m0 + j0) * g.ldc + n;
                if (SPLIT) {
                    // partial tile [NB][WR] over the stages, which nothing reads or fills any more: this part's blocks are all multiplied
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        sts32(sbase + 4u * (uint32_t)((j0 + j) * WR + 32 * h + lane), nkb ? (int)r[j] : 0);
                } else if (n < g.N) {
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        if (j0 + j < rows) store_value(g.C, at + j * g.ldc, g.c_type, __uint_as_float(r[j]) * f);
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_tempty(acc));
            aph ^= acc;
            acc ^= 1u;
        }
    }
    __syncwarp();
    tc_fence_before();
    if (SPLIT) cluster_sync_all();           // every partial tile is written
    else __syncthreads();
    tc_fence_after();
    if (warp == 1)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)C::COLS) : "memory");
    if (SPLIT) {
        // one tile per cluster: each CTA adds its share of the rows of all partial tiles, in order
        if (walk.get(first, t)) {
            const float f = (g.FA ? __ldg(g.FA) : 1.0f) * (g.FB ? __ldg(g.FB + t.e) : 1.0f);
            const int rows = min(NB, t.m_end - t.m0), lo = rows * split / splits, hi = rows * (split + 1) / splits;
            const int n = t.n0 + 4 * lane, have = min(4, g.N - n);
            for (int m = lo + warp; m < hi; m += FEW_THREADS / 32) {
                float4 q[MAX_SPLITS];
#pragma unroll
                for (int s = 0; s < MAX_SPLITS; ++s) {
                    q[s] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                    if (s < splits) q[s] = lds128_cluster(map_to_cta(sbase + (uint32_t)((m * WR + 4 * lane) * 4), (uint32_t)s));
                }
                float v[4] = {};
#pragma unroll
                for (int s = 0; s < MAX_SPLITS; ++s) {
                    v[0] += q[s].x;
                    v[1] += q[s].y;
                    v[2] += q[s].z;
                    v[3] += q[s].w;
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] *= f;
                const int64_t at = (int64_t)(t.m0 + m) * g.ldc + n;
                if (p.c_vec && have == 4) {
                    if (g.c_type == Q4_F32)
                        *reinterpret_cast<float4*>(static_cast<float*>(g.C) + at) = make_float4(v[0], v[1], v[2], v[3]);
                    else
                        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(g.C) + at) =
                            g.c_type == Q4_BF16 ? make_uint2(f8::pack2(v[0], v[1], (const __nv_bfloat16*)nullptr), f8::pack2(v[2], v[3], (const __nv_bfloat16*)nullptr))
                                                : make_uint2(f8::pack2(v[0], v[1], (const __half*)nullptr), f8::pack2(v[2], v[3], (const __half*)nullptr));
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (j < have) store_value(g.C, at + j, g.c_type, v[j]);
                }
            }
        }
        cluster_sync_all();                  // the partial tiles have been read
    }
}

template <int NB, bool BY16, bool SPLIT>
static q4_status launch_few(FewParams& p, int64_t tiles, cudaStream_t st)
{
    using Cf = FewCfg<NB, BY16>;
    auto kernel = gemm_f4_few_kernel<NB, BY16, SPLIT>;
    const GemmParams& g = p.g;
    const int kbytes = (g.K + 1) / 2;
    CUtensorMap a, b;
    if (!make_byte_map(&a, g.A, g.lda, g.M, kbytes, NB) ||
        !make_byte_map(&b, g.Bt, g.ldb, (int)((int64_t)g.N * (g.E ? g.E : 1)), kbytes, WR)) return Q4_ERR_CUDA;
    static bool ready[64] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return Q4_ERR_CUDA;
    if (!ready[dev]) {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Cf::SMEM) != cudaSuccess) return Q4_ERR_CUDA;
        ready[dev] = true;
    }
    const int64_t sms = 2 * f8_pairs_of_device();
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)p.splits;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(SPLIT ? tiles * p.splits : tiles < sms ? tiles : sms));
    cfg.blockDim = dim3(FEW_THREADS);
    cfg.dynamicSmemBytes = Cf::SMEM;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = SPLIT ? 2 : 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, a, b, p);
    count_launch();
    return e == cudaSuccess ? Q4_OK : Q4_ERR_CUDA;
}

template <int NB, bool BY16>
static q4_status launch_nb(FewParams& p, int64_t tiles, cudaStream_t st)
{
    return p.splits > 1 ? launch_few<NB, BY16, true>(p, tiles, st) : launch_few<NB, BY16, false>(p, tiles, st);
}

}  // namespace f4

using namespace f4;

// Parts of the depth of a dense product of `tiles` tiles: twice as many while the clusters fit the device at once (a cluster
// lies within a GPC, so 33 of four CTAs and 15 of eight fit where 148 SMs do) and a part keeps two stages.
static int few_splits(int64_t tiles, int blocks)
{
    int splits = 1;
    while (splits < MAX_SPLITS && 2 * splits * tiles <= 2 * f8_pairs_of_device() * 8 / 10 + (splits == 1 ? 8 : splits == 2 ? 14 : 2) && blocks >= 4 * splits)
        splits *= 2;
    return splits;
}

// Where it pays: by experts up to 64 rows per expert on average; one product up to 128 rows, and more while its tiles are so
// few that the depth in parts saves more (500 clk per stage that another part takes) than the exchange costs (300 x 300 x
// 2000 6.5 us against 7.6 on pairs, 500 x 500 x 2048 6.5 against 7.2, 200 x 250 x 1024 6.5 against 6.0).
bool gemm_f4_few_supported(const f4::GemmParams& g)
{
    if ((uintptr_t)g.A % 16 || (uintptr_t)g.Bt % 16 || g.lda % 16 || g.ldb % 16) return false;
    if (g.M >= INT32_MAX - 512 || (int64_t)g.N * (g.E ? g.E : 1) >= INT32_MAX - 512) return false;
    if (g.E) return g.M <= 64 * (int64_t)g.E;
    if (g.M <= 128) return true;
    const int64_t tiles = ((int64_t)g.M + 127) / 128 * (((int64_t)g.N + WR - 1) / WR);
    const int blocks = (g.K + STAGE_K - 1) / STAGE_K, splits = few_splits(tiles, blocks);
    return tiles <= 16 && (blocks - (blocks + splits - 1) / splits) * 500 > 2500;
}

q4_status launch_gemm_f4_few(const f4::GemmParams& g, bool by16, cudaStream_t st)
{
    FewParams p{};
    p.g = g;
    const size_t es = f8::type_size(g.c_type);
    p.c_vec = (uintptr_t)g.C % (4 * es) == 0 && g.ldc % 4 == 0;
    // columns: what holds the rows, or twice an expert's average
    const int64_t want = g.E ? 2 * ((int64_t)g.M / g.E) : g.M;
    const int nb = want <= 16 ? 16 : want <= 32 ? 32 : want <= 64 ? 64 : 128;
    p.tiles_m = (int)(((int64_t)g.M + nb - 1) / nb);
    p.tiles_n = (int)(((int64_t)g.N + WR - 1) / WR);
    const int64_t tiles = (p.tiles_m + (g.E ? (g.E < g.M ? g.E : g.M) : 0)) * (int64_t)p.tiles_n;
    p.splits = g.E ? 1 : few_splits(tiles, (g.K + STAGE_K - 1) / STAGE_K);
    switch (nb) {
    case 16: return by16 ? launch_nb<16, true>(p, tiles, st) : launch_nb<16, false>(p, tiles, st);
    case 32: return by16 ? launch_nb<32, true>(p, tiles, st) : launch_nb<32, false>(p, tiles, st);
    case 64: return by16 ? launch_nb<64, true>(p, tiles, st) : launch_nb<64, false>(p, tiles, st);
    default: return by16 ? launch_nb<128, true>(p, tiles, st) : launch_nb<128, false>(p, tiles, st);
    }
}

}  // namespace q4
