// e4m3 product with block scales for few rows of A (tokens being decoded): every weight is read once and
// the weights' stream never pauses.
//
//   C[m][n] = sum over blocks b of 128 depth values of  SA[b][m] * SB(n, b) * sum_k a(m, k) b(n, k)
//
// One persistent CTA per SM walks tiles of 16 * R rows of Bt (output columns) by up to MB (16 or 32) rows of A of one
// expert.  Producer warps keep a ring of stages filled by TMA, a block of depth per stage: the tile's rows of Bt,
// MB rows of A (128-byte swizzle) and their scales (4-byte asynchronous copies), tile after tile without a
// break.  Eight consumer warps take the stages in turn: warp-level matrix instructions (16 x 8 x 32) with
// Bt's rows as their 16 and the rows of A as their 8, scaled binary32 sums in registers, which are added over the
// warps, in order, at the tile's end while the next tiles' stages arrive.
// The order of depth values inside a block is free as long as both operands share it: lane (g, t) takes
// 16-byte pieces 2 t and 2 t + 1 of its rows, which the swizzle spreads over all banks.
// Bound: HBM; the tensor memory kernel would drain a 128-row accumulator per block for a handful of rows.
// 64 experts of 2048 x 1024, 16 tokens x 8: 22 us = 5.4 TB/s of weights (pair kernel 34 us); one token through
// 4096 x 4096: 5.9 us in a graph, of which the weights take 2.6.
#include <cuda.h>

#include "q4_f8.cuh"
#include "q4_tc_ptx.cuh"

namespace q4 {

bool make_byte_map(CUtensorMap* tm, const uint8_t* base, int64_t ld, int rows, int kbytes, int box_rows);

namespace f8 {

constexpr int CONSUMERS = 8;

// R: groups of 16 rows of Bt per tile; MB: rows of A per tile (16 or 32).
template <int R, int MB> struct FewCfg {
    static constexpr int NB = 16 * R;                          // rows of Bt per tile
    // A stage's waits, copies and arrivals take a producer warp about 500 clk, two to four times what its bytes
    // take: four warps in turn, eight for the smallest stage (16384 x 4096: 17.5 -> 15.1 us; they cost
    // the others registers: 64 experts 22 -> 23 us)
    static constexpr int PRODUCERS = R == 2 && MB == 16 ? 8 : 4;
    static constexpr int STAGE = (NB + MB) * BLK;
    // Stage s is always filled by producer s % PRODUCERS and emptied by consumer s % CONSUMERS: a wait on a
    // barrier's parity is only right for a warp that has seen the round before.
    static constexpr int STAGES = R == 4 || MB == 32 ? 16 : 24;
    static_assert(STAGES % PRODUCERS == 0 && STAGES % CONSUMERS == 0, "a stage belongs to one producer and one consumer");
    static constexpr int OFF_SCALE = STAGES * STAGE;           // per stage: MB SA, 64 SB
    static constexpr int SCALE = (MB + 64) * 4;
    static constexpr int OFF_PART = OFF_SCALE + STAGES * SCALE;
    static constexpr int PITCH = NB + 4;
    static constexpr int PART = CONSUMERS * MB * PITCH * 4;
    static constexpr int PARTS = R == 4 ? 1 : 2;               // two take turns where they fit
    static constexpr int OFF_CUM = OFF_PART + PARTS * PART;        // tiles before each expert
    static constexpr int OFF_BAR = OFF_CUM + (Q4_MAX_EXPERTS + 32) * 4;
    static constexpr int OFF_MISC = OFF_BAR + 2 * STAGES * 8;
    static constexpr int SMEM = OFF_MISC + 16 + 1024;
    static_assert(STAGE % 1024 == 0 && SMEM <= 232448, "shared memory");
};

__device__ __forceinline__ void mma_e4m3(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
                 "{%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void copy_scale(uint32_t dst, const float* src, bool in)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(in ? 4 : 0) : "memory");
}

struct FewTile { int e, n0, m0, rows; };

// Tile t of the walk, by a whole warp: the expert whose tiles cover it (cum: tiles before each expert, E padded to
// a multiple of 32 with the total), then row groups fastest, so that they share the weights in L2.
template <int R, int MB>
__device__ __forceinline__ FewTile few_tile(const GemmF8Params& p, uint32_t cum_s, int t, int lane)
{
    constexpr int NB = 16 * R;
    FewTile f;
    int lo = 0, hi = p.M;
    f.e = 0;
    int local = t;
    if (p.mode == kExpertRows) {
        const int blocks = (p.E + 31) / 32;
        const int b = __popc(__ballot_sync(0xFFFFFFFFu, lane < blocks && lds32(cum_s + 4u * (uint32_t)(lane < blocks ? lane * 32 : 0)) <= t)) - 1;
        const int c = lds32(cum_s + 4u * (uint32_t)(b * 32 + lane));
        const int i = __popc(__ballot_sync(0xFFFFFFFFu, c <= t)) - 1;
        f.e = b * 32 + i;
        local = t - __shfl_sync(0xFFFFFFFFu, c, i);
        lo = min(max(p.starts[f.e], 0), p.M);
        hi = min(max(p.starts[f.e + 1], lo), p.M);
    }
    const int groups = (hi - lo + MB - 1) / MB, n = local / groups;
    f.n0 = n * NB;
    f.m0 = lo + (local - n * groups) * MB;
    f.rows = min(MB, hi - f.m0);
    return f;
}

template <int R, int MB>
__global__ void __launch_bounds__((CONSUMERS + FewCfg<R, MB>::PRODUCERS) * 32, 1)
gemm_f8_few_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const GemmF8Params p)
{
    using C = FewCfg<R, MB>;
    constexpr int NB = C::NB, NT = MB / 8;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t sbase = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t cum_s = sbase + C::OFF_CUM, bar0 = sbase + C::OFF_BAR, abort_flag = sbase + C::OFF_MISC;
    auto bar_full  = [&](int s) { return bar0 + 8u * (uint32_t)s; };
    auto bar_empty = [&](int s) { return bar0 + 8u * (uint32_t)(C::STAGES + s); };
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int ntn = (p.N + NB - 1) / NB, nkb = (p.K + BLK - 1) / BLK;

    if (threadIdx.x == 0) {
        for (int s = 0; s < C::STAGES; ++s) {
            mbar_init(bar_full(s), 1 + 32);        // the copies' announcement, and each producer lane's scales
            mbar_init(bar_empty(s), 1);
        }
        sts32(abort_flag, 0);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async_smem();
    }
    wait_for_predecessor();
    int ntiles = (p.M + MB - 1) / MB * ntn;
    if (p.mode == kExpertRows) {
        if (warp == 0) {
            int at = 0;
            for (int e0 = 0; e0 < p.E; e0 += 32) {
                const int e = e0 + lane;
                int s = 0;
                if (e < p.E) {
                    const int lo = min(max(p.starts[e], 0), p.M), hi = min(max(p.starts[e + 1], lo), p.M);
                    s = (hi - lo + MB - 1) / MB * ntn;
                }
                const int own = s;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int v = __shfl_up_sync(0xFFFFFFFFu, s, o);
                    if (lane >= o) s += v;
                }
                // an expert without tiles repeats the next one's number and is never the last that is <= t
                sts32(cum_s + 4u * (uint32_t)e, e < p.E ? at + s - own : INT32_MAX);
                at += __shfl_sync(0xFFFFFFFFu, s, 31);
            }
            if (lane == 0) sts32(abort_flag + 4, at);
        }
    }
    __syncthreads();
    if (p.mode == kExpertRows) ntiles = lds32(abort_flag + 4);

    if (warp >= CONSUMERS) {
        // ------------------------------------------------------------ producer
        int it = 0;
        for (int tile = blockIdx.x; tile < ntiles; tile += gridDim.x) {
            const FewTile f = few_tile<R, MB>(p, cum_s, tile, lane);
            const int64_t brow = (int64_t)f.e * p.N + f.n0;
            const float* sb = p.b_rows ? p.SB + f.n0 + lane : p.SB + (f.e * blocks_of(p.N) + f.n0 / BLK) * p.ldsb;
            const float* sa = p.SA + f.m0 + lane;
            for (int b = 0; b < nkb; ++b, ++it) {
                if ((it & (C::PRODUCERS - 1)) != warp - CONSUMERS) continue;
                const int st = it % C::STAGES;
                mbar_wait_suspend(bar_empty(st), ((uint32_t)(it / C::STAGES) & 1u) ^ 1u, abort_flag, p.status);
                const uint32_t dst = sbase + st * C::STAGE, sc = sbase + C::OFF_SCALE + st * C::SCALE;
                if (elect_one()) {
                    mbar_expect_tx(bar_full(st), (uint32_t)C::STAGE);
                    tma_load_2d(dst, &tmB, b * BLK, (int)brow, bar_full(st));
                    tma_load_2d(dst + NB * BLK, &tmA, b * BLK, f.m0, bar_full(st));
                }
                __syncwarp();
                if (lane < MB) copy_scale(sc + 4u * (uint32_t)lane, lane < f.rows ? sa + b * p.ldsa : p.SA, lane < f.rows);
                if (p.b_rows) {
#pragma unroll
                    for (int i = 0; i < NB / 32; ++i)
                        copy_scale(sc + 4u * (uint32_t)(MB + lane + 32 * i), f.n0 + lane + 32 * i < p.N ? sb + b * p.ldsb + 32 * i : p.SB,
                                   f.n0 + lane + 32 * i < p.N);
                } else if (lane == 0) {
                    copy_scale(sc + 4u * MB, sb + b, true);
                }
                asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar_full(st)) : "memory");
            }
            if (lds32(abort_flag)) break;
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        return;
    }
    // ---------------------------------------------------------------- consumers
    const int g = lane >> 2, t = lane & 3;
    const uint32_t p0 = (uint32_t)(g * BLK + (((2 * t) ^ g) << 4)), p1 = (uint32_t)(g * BLK + (((2 * t + 1) ^ g) << 4));
    int first = 0, buf = 0;                       // stage (over all tiles) of the tile's first block
    for (int tile = blockIdx.x; tile < ntiles; tile += gridDim.x, first += nkb, buf ^= 1) {
        const FewTile f = few_tile<R, MB>(p, cum_s, tile, lane);
        float acc[R][NT][4] = {};
        for (int b = (warp - first) & (CONSUMERS - 1); b < nkb; b += CONSUMERS) {
            const int it = first + b, st = it % C::STAGES;
            mbar_wait_suspend(bar_full(st), (uint32_t)(it / C::STAGES) & 1u, abort_flag, p.status);
            const uint32_t ws = sbase + st * C::STAGE, as = ws + NB * BLK, sc = sbase + C::OFF_SCALE + st * C::SCALE;
            uint4 a[NT][2];
            float sa[NT][2];
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                a[j][0] = lds128(as + 8 * j * BLK + p0);
                a[j][1] = lds128(as + 8 * j * BLK + p1);
                sa[j][0] = __int_as_float(lds32(sc + 4u * (uint32_t)(8 * j + 2 * t)));
                sa[j][1] = __int_as_float(lds32(sc + 4u * (uint32_t)(8 * j + 2 * t + 1)));
            }
            const float sb = __int_as_float(lds32(sc + 4u * MB));
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const uint4 u0 = lds128(ws + 16 * r * BLK + p0), u1 = lds128(ws + 16 * r * BLK + p1);
                const uint4 v0 = lds128(ws + (16 * r + 8) * BLK + p0), v1 = lds128(ws + (16 * r + 8) * BLK + p1);
                float s0 = sb, s1 = sb;
                if (p.b_rows) {
                    s0 = __int_as_float(lds32(sc + 4u * (uint32_t)(MB + 16 * r + g)));
                    s1 = __int_as_float(lds32(sc + 4u * (uint32_t)(MB + 16 * r + 8 + g)));
                }
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    if (8 * j >= f.rows) break;
                    float d[4] = {};
                    mma_e4m3(d, u0.x, v0.x, u0.y, v0.y, a[j][0].x, a[j][0].y);
                    mma_e4m3(d, u0.z, v0.z, u0.w, v0.w, a[j][0].z, a[j][0].w);
                    mma_e4m3(d, u1.x, v1.x, u1.y, v1.y, a[j][1].x, a[j][1].y);
                    mma_e4m3(d, u1.z, v1.z, u1.w, v1.w, a[j][1].z, a[j][1].w);
                    acc[r][j][0] = fmaf(d[0] * s0, sa[j][0], acc[r][j][0]);
                    acc[r][j][1] = fmaf(d[1] * s0, sa[j][1], acc[r][j][1]);
                    acc[r][j][2] = fmaf(d[2] * s1, sa[j][0], acc[r][j][2]);
                    acc[r][j][3] = fmaf(d[3] * s1, sa[j][1], acc[r][j][3]);
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_empty(st));
        }
        // partial sums [warp][row of A][row of Bt]; the barrier of the next tile tells that these have been read
        if (C::PARTS == 1) asm volatile("bar.sync 1, 256;" ::: "memory");       // the last tile's have been read
        const uint32_t part = sbase + C::OFF_PART + (uint32_t)((C::PARTS == 1 ? 0 : buf) * C::PART);
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            if (8 * j >= f.rows) break;
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    sts32(part + 4u * (uint32_t)((warp * MB + 8 * j + 2 * t + (i & 1)) * C::PITCH + 16 * r + 8 * (i >> 1) + g),
                          __float_as_int(acc[r][j][i]));
        }
        asm volatile("bar.sync 1, 256;" ::: "memory");
        for (int u = threadIdx.x; u < f.rows * NB; u += CONSUMERS * 32) {
            const int m = u / NB, n = u % NB;
            if (f.n0 + n >= p.N) continue;
            float v = 0.0f;
#pragma unroll
            for (int k = 0; k < CONSUMERS; ++k) v += __int_as_float(lds32(part + 4u * (uint32_t)((k * MB + m) * C::PITCH + n)));
            const int64_t at = (int64_t)(f.m0 + m) * p.ldc + f.n0 + n;
            if (p.c_type == Q4_F32) static_cast<float*>(p.C)[at] = v;
            else if (p.c_type == Q4_BF16) static_cast<__nv_bfloat16*>(p.C)[at] = __float2bfloat16_rn(v);
            else static_cast<__half*>(p.C)[at] = __float2half_rn(v);
        }
    }
}

template <int R, int MB>
static q4_status launch_few(const GemmF8Params& p, int64_t tiles, int sms, cudaStream_t st)
{
    using C = FewCfg<R, MB>;
    CUtensorMap a, b;
    if (!make_byte_map(&a, p.A, p.lda, p.M, p.K, MB) ||
        !make_byte_map(&b, p.Bt, p.ldb, (int)(p.mode == kExpertRows ? (int64_t)p.E * p.N : p.N), p.K, C::NB)) return Q4_ERR_CUDA;
    static bool ready[64] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return Q4_ERR_CUDA;
    if (!ready[dev]) {
        if (cudaFuncSetAttribute(gemm_f8_few_kernel<R, MB>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM) != cudaSuccess)
            return Q4_ERR_CUDA;
        ready[dev] = true;
    }
    const cudaError_t e = launch(gemm_f8_few_kernel<R, MB>, (unsigned)(tiles < sms ? tiles : sms), (CONSUMERS + C::PRODUCERS) * 32,
                                 C::SMEM, st, a, b, p);
    return e == cudaSuccess ? Q4_OK : Q4_ERR_CUDA;
}

}  // namespace f8

using namespace f8;

// Where it pays (measured, 148 SMs): by experts up to 8 rows per expert on average (64 experts of 2048 x 1024: 512
// rows 34 against 43 us on the pair kernel, 1024 rows 55 against 43); one product up to 16 rows (4096 x 4096: 6.6
// against 10.7 us), and up to 32 while its tiles go round the SMs twice at most (4096 x 4096 8.2 against 11.6 us,
// 16384 x 4096 26 against 22 us): beyond, the warp-level matrix instructions bind.
// By experts the rule knows the rows of A's buffer, not the segments, which are on the device.  Where they are not alike, it
// can choose the slower kernel: 512 rows all at one of 64 experts take 19 us here, 8 on the pair kernel (64 rows 4.8 and
// 7.3); a buffer of more rows than its segments hold goes to the pair kernel (a serving sort leaves none: align = 1).
bool gemm_f8_few_supported(const GemmF8Params& g)
{
    if ((uintptr_t)g.A % 16 || (uintptr_t)g.Bt % 16 || g.lda % 16 || g.ldb % 16) return false;
    if ((int64_t)g.N * (g.mode == kExpertRows ? g.E : 1) >= INT32_MAX - 512) return false;
    if (g.mode == kExpertRows) return g.M <= 8 * (int64_t)g.E;
    return g.mode == kDense && (g.M <= 16 || (g.M <= 32 && ((int64_t)g.N + 31) / 32 <= 4 * f8_pairs_of_device()));
}

q4_status launch_gemm_f8_few(const GemmF8Params& p, cudaStream_t st)
{
    const int sms = 2 * f8_pairs_of_device();
    if (p.mode == kDense && p.M > 16) return launch_few<2, 32>(p, ((int64_t)p.N + 31) / 32, sms, st);
    const int64_t groups = ((int64_t)p.M + 15) / 16 + (p.mode == kExpertRows ? (p.E < p.M ? p.E : p.M) : 0);
    // 64 columns per tile where the tiles still go round the SMs a few times (half the stages' overhead per
    // byte: 50 experts 22 against 27 us); else 32
    const int64_t t64 = groups * (((int64_t)p.N + 63) / 64), t32 = groups * (((int64_t)p.N + 31) / 32);
    return t64 >= 4 * sms ? launch_few<4, 16>(p, t64, sms, st) : launch_few<2, 16>(p, t32, sms, st);
}

}  // namespace q4
