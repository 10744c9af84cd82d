// Expert layer for a few tokens on e2m1 weights with microscales: two kernels that stream the weights of the experts that
// are hit, once, from HBM.
//
//   kernel 1 (up)     h = silu(G_e x) * (U_e x)  (or silu(G_e x)) of every pair of a token and an expert, binary32
//   kernel 2 (down)   y = W2_e h of every pair, binary32; the block that finishes a tile of columns last sums
//                     Out[t] = sum_j w[t][j] y in the order of j
//
// Every block sorts the pairs by expert for itself (a few hundred numbers).  A unit is up to 8 * NT pairs of one expert, a
// tile 64 rows of its weights (gated: 32 of G and the same 32 of U).  One persistent block per SM walks tiles, a
// unit's one after the other, so that the unit's activations stay in shared memory:
//
//   warps 8..11  producers   a stage (256 depth values) of the tile's rows by TMA (128-byte swizzle), its words of scales
//                            by 4-byte asynchronous copies, tile after tile without a break
//   warps 0..7   consumers   in turn a stage each: codes become binary16 numbers, warp-level matrix instructions (16 x 8 x 16)
//                            with the weights' rows as their 16 and the pairs as their 8, binary32 sums in registers,
//                            which are added over the warps, in order, at the tile's end
//
// Activations are held in binary16, a row times a power of two that takes its largest value to 2^14 .. 2^15.  That is
// exact for binary16 and bfloat16 values down to 2^-38 of a row's largest; h, computed in binary32, is rounded to
// 11 bits by it (an eighth of a step of a bfloat16 output).
//
// The order of depth values inside a stage is free as long as both operands share it, and is chosen for the scales: BY16 a
// lane holds 64 consecutive values of a row, whose four scales are one word, and a code times its scale is exact in
// binary16; else the four lanes of a row share a group of 32, whose two products are scaled in binary32.
// Bound: HBM, with instruction issue next (about 14 instructions for 128 bytes of codes by 16, 11 by 32).
#include <cuda.h>

#include "q4_f4.cuh"
#include "q4_tc_ptx.cuh"

namespace q4 {

bool make_byte_map(CUtensorMap* tm, const uint8_t* base, int64_t ld, int rows, int kbytes, int box_rows);

namespace f4 {

constexpr int CONSUMERS = 8, PRODUCERS = 4;
constexpr int LAYER_THREADS = (CONSUMERS + PRODUCERS) * 32;
constexpr int TROWS = 64, BOXROWS = 32;          // weights' rows of a tile and of a copy
constexpr int SK = 256, SROWB = 128;             // depth values and bytes per row of a stage
constexpr int MAX_PAIRS = 1024;                  // sorted by each block

// Shared memory, in this order: stages, their scales, pairs' activations, partial sums, the sorted pairs, barriers.
template <bool BY16, int NT> struct LayerCfg {
    static constexpr int WORDS = BY16 ? 4 : 2;
    static constexpr int STAGE = TROWS * SROWB;
    static constexpr int SCALE = WORDS * TROWS * 4;
    static constexpr int N = 8 * NT;                           // pairs of a unit
    static constexpr int PITCH = TROWS + 4;
    static constexpr int PART = CONSUMERS * N * PITCH * 4;
    static constexpr int LISTS = MAX_PAIRS * 2 * 3 + (Q4_MAX_EXPERTS + 32) * 4 * 2;
    static constexpr int TAIL = 2 * 16 * 8 + 64 + N * 8;       // barriers, words, pairs' scales
    static __host__ __device__ constexpr int act_pitch(int nkb) { return nkb * SK * 2 + 64; }
    static __host__ __device__ constexpr int bytes(int stages, int nkb)
    {
        return stages * (STAGE + SCALE) + N * act_pitch(nkb) + PART + LISTS + TAIL + 1024;
    }
};

struct LayerLaunch {
    LayerParams p;
    float* hidden;                   // [pairs][H]
    float* y;                        // [pairs][D]
    int* done;                       // per tile of output columns
    int stages;
};

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
                 "{%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t mul2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// the binary16 values of two e4m3 numbers
__device__ __forceinline__ uint32_t scales2(uint32_t bytes)
{
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)bytes));
    return r;
}
__device__ __forceinline__ void copy_word(uint32_t dst, const uint32_t* src, bool in)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(in ? 4 : 0) : "memory");
}
__device__ __forceinline__ void sync_consumers() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

// Sorts the pairs by expert: order[] = pairs, expert by expert, in their own order; units of up to N pairs.  All threads.
template <int N>
__device__ __forceinline__ int sort_pairs(const LayerParams& p, uint16_t* order, uint16_t* rank, uint16_t* unit, int* first, int* units, int* total)
{
    const int n = p.tokens * p.topk, lane = threadIdx.x & 31, padded = (p.E + 31) & ~31;
    for (int e = threadIdx.x; e < padded; e += LAYER_THREADS) first[e] = 0;
    __syncthreads();
    if (threadIdx.x < 32) {
        for (int i0 = 0; i0 < n; i0 += 32) {
            const int i = i0 + lane, e = i < n ? __ldg(p.ids + i) : -1;
            const bool in = (unsigned)e < (unsigned)p.E;
            const unsigned same = __match_any_sync(0xFFFFFFFFu, in ? e : -1), before = same & ((1u << lane) - 1u);
            const int have = in ? first[e] : 0;
            __syncwarp();
            if (in) {
                rank[i] = (uint16_t)(have + __popc(before));
                if (!before) first[e] = have + __popc(same);
            }
            __syncwarp();
        }
        int at = 0, un = 0;
        for (int e0 = 0; e0 < padded; e0 += 32) {
            const int c = first[e0 + lane], u = (c + N - 1) / N;
            int sc = c, su = u;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int a = __shfl_up_sync(0xFFFFFFFFu, sc, o), b = __shfl_up_sync(0xFFFFFFFFu, su, o);
                if (lane >= o) { sc += a; su += b; }
            }
            first[e0 + lane] = at + sc - c;
            units[e0 + lane] = un + su - u;
            for (int k = 0; k < u; ++k) unit[un + su - u + k] = (uint16_t)(e0 + lane);
            at += __shfl_sync(0xFFFFFFFFu, sc, 31);
            un += __shfl_sync(0xFFFFFFFFu, su, 31);
        }
        if (lane == 0) {
            first[padded] = at;
            *total = un;
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += LAYER_THREADS) {
        const int e = __ldg(p.ids + i);
        if ((unsigned)e < (unsigned)p.E) order[first[e] + rank[i]] = (uint16_t)i;
    }
    __syncthreads();
    return *total;
}

// A pair's activations (or hidden values) to shared memory as binary16 numbers times a power of two, in the stage's order;
// by a warp.  Returns the power's inverse.
template <bool BY16, typename T>
__device__ __forceinline__ float put_activations(const T* row, int K, int nkb, uint32_t dst, int lane)
{
    const bool vec = (uintptr_t)row % 16 == 0;
    auto eight = [&](int k, float (&v)[8]) {
        if (vec && k + 8 <= K) {
            f8::Eight<T> e;
#pragma unroll
            for (int q = 0; q < f8::Eight<T>::NW / 4; ++q) {
                const uint4 u = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint8_t*>(row + k) + 16 * q);
                e.w[4 * q] = u.x; e.w[4 * q + 1] = u.y; e.w[4 * q + 2] = u.z; e.w[4 * q + 3] = u.w;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = e.get(i);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = k + i < K ? f8::to_f(row[k + i]) : 0.0f;
        }
    };
    uint32_t a = 0;
#pragma unroll 4
    for (int k = lane * 8; k < K; k += 256) {
        float v[8];
        eight(k, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) a = max(a, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    }
    a = __reduce_max_sync(0xFFFFFFFFu, a);
    // a row that is not finite keeps its values
    const uint32_t e = a == 0 || a >= 0x7F800000u ? 141u : max(a >> 23, 15u);
    const float s = __uint_as_float((268u - e) << 23);
#pragma unroll 4
    for (int b = 0; b < nkb; ++b) {
        float v[8];
        eight(b * SK + lane * 8, v);
        uint32_t h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = f8::pack2(v[2 * i] * s, v[2 * i + 1] * s, (const __half*)nullptr);
        // BY16: value 64 t + 8 i + r of the stage lies at 16 bytes t of piece i
        const int at = BY16 ? (lane & 7) * 64 + (lane >> 3) * 16 : lane * 16;
        sts128(dst + (uint32_t)(b * SK * 2 + at), make_uint4(h[0], h[1], h[2], h[3]));
    }
    return __uint_as_float((e - 14u) << 23);
}

template <bool BY16, int NT, bool DOWN>
__global__ void __launch_bounds__(LAYER_THREADS, 1)
layer_kernel(const __grid_constant__ CUtensorMap tmW, const LayerLaunch L)
{
    using C = LayerCfg<BY16, NT>;
    const LayerParams& p = L.p;
    extern __shared__ uint8_t smem_raw[];
    const int K = DOWN ? p.H : p.D, nkb = (K + SK - 1) / SK, pitch = C::act_pitch(nkb), STAGES = L.stages;
    const uint32_t sbase = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t scales_s = sbase + STAGES * C::STAGE, act_s = scales_s + STAGES * C::SCALE, part_s = act_s + C::N * pitch,
                   lists_s = part_s + C::PART, tail_s = lists_s + C::LISTS;
    uint8_t* const lists = smem_raw + (lists_s - smem_u32(smem_raw));
    int* const first = reinterpret_cast<int*>(lists);                       // [E, a multiple of 32, + 1]
    int* const units = first + Q4_MAX_EXPERTS + 32;                         // units before each expert
    uint16_t* const order = reinterpret_cast<uint16_t*>(units + Q4_MAX_EXPERTS + 32);
    uint16_t* const rank = order + MAX_PAIRS;
    uint16_t* const unit = rank + MAX_PAIRS;                                // expert of each unit
    int* const words = reinterpret_cast<int*>(smem_raw + (tail_s + 2 * 16 * 8 - smem_u32(smem_raw)));
    float* const inverse = reinterpret_cast<float*>(words + 16);            // [N]
    auto bar_full  = [&](int s) { return tail_s + 8u * (uint32_t)s; };
    auto bar_empty = [&](int s) { return tail_s + 8u * (uint32_t)(16 + s); };
    const uint32_t abort_flag = tail_s + 2 * 16 * 8;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(bar_full(s), 1 + 32);        // the copies' announcement, and each producer lane's scales
            mbar_init(bar_empty(s), 1);
        }
        words[0] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async_smem();
    }
    // Kernel 2 starts when every block of kernel 1 has waited for what came before them: what it reads but for the
    // hidden values is there, and its bounded waits ahead of those last as long as kernel 1 at most.
    if (!DOWN) f8::wait_for_predecessor();
    const int nunits = sort_pairs<C::N>(p, order, rank, unit, first, units, words + 1);
    const int rows = DOWN ? p.D : p.H;                          // of the output
    const int per_tile = !DOWN && p.gated ? TROWS / 2 : TROWS;
    const int ntr = (rows + per_tile - 1) / per_tile, ntiles = nunits * ntr;
    if (!DOWN)
        for (int i = blockIdx.x * LAYER_THREADS + threadIdx.x; i < (p.D + TROWS - 1) / TROWS; i += gridDim.x * LAYER_THREADS) L.done[i] = 0;
    // a block's tiles lie together
    const int t0 = (int)((int64_t)ntiles * blockIdx.x / gridDim.x), t1 = (int)((int64_t)ntiles * (blockIdx.x + 1) / gridDim.x);
    const int64_t wrows = (int64_t)p.E * (DOWN ? p.D : p.gated ? 2 * p.H : p.H);

    if (warp >= CONSUMERS) {
        // ------------------------------------------------------------ producers
        const uint32_t* const S = DOWN ? p.S2 : p.S1;
        const int64_t lds = DOWN ? p.lds2 : p.lds1;
        const int nw = (int)words_of(K, BY16);
        int it = 0;
        for (int tile = t0; tile < t1; ++tile) {
            const int u = tile / ntr, r0 = (tile - u * ntr) * per_tile;
            const int64_t ra = (int64_t)unit[u] * (wrows / p.E) + r0, rb = ra + (!DOWN && p.gated ? p.H : BOXROWS);
            for (int b = 0; b < nkb; ++b, ++it) {
                if ((it & (PRODUCERS - 1)) != warp - CONSUMERS) continue;
                const int st = it % STAGES;
                mbar_wait_suspend(bar_empty(st), ((uint32_t)(it / STAGES) & 1u) ^ 1u, abort_flag, p.status);
                const uint32_t dst = sbase + st * C::STAGE, sc = scales_s + st * C::SCALE + 4u * (uint32_t)lane;
                if (elect_one()) {
                    mbar_expect_tx(bar_full(st), (uint32_t)C::STAGE);
                    tma_load_2d(dst, &tmW, b * SROWB, (int)ra, bar_full(st));
                    tma_load_2d(dst + BOXROWS * SROWB, &tmW, b * SROWB, (int)rb, bar_full(st));
                }
                __syncwarp();
#pragma unroll
                for (int w = 0; w < C::WORDS; ++w) {
                    const bool in = b * C::WORDS + w < nw;
                    const uint32_t* const src = S + (in ? (b * C::WORDS + w) * lds : 0);
                    const bool ia = in && ra + lane < wrows, ib = in && rb + lane < wrows;
                    copy_word(sc + (uint32_t)(w * TROWS * 4), ia ? src + ra + lane : S, ia);
                    copy_word(sc + (uint32_t)((w * TROWS + BOXROWS) * 4), ib ? src + rb + lane : S, ib);
                }
                asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar_full(st)) : "memory");
            }
            if (lds32(abort_flag)) break;
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        return;
    }
    // ---------------------------------------------------------------- consumers
    if (DOWN) f8::wait_for_predecessor();                      // the hidden values, and the counters' zeros
    const int g = lane >> 2, t = lane & 3;
    int at_unit = -1, begin = 0, count = 0, it0 = 0;
    float f = 1.0f;
    for (int tile = t0; tile < t1; ++tile, it0 += nkb) {
        const int u = tile / ntr, r0 = (tile - u * ntr) * per_tile;
        if (u != at_unit) {
            at_unit = u;
            const int e = unit[u];
            begin = first[e] + (u - units[e]) * C::N;
            count = min(C::N, first[e + 1] - begin);
            const float* const F = DOWN ? p.F2 : p.F1;
            f = F ? __ldg(F + e) : 1.0f;
            // (the tile before ended with a barrier behind its last reading of activations)
            for (int n = warp; n < count; n += CONSUMERS) {
                const int pair = order[begin + n];
                const uint32_t dst = act_s + (uint32_t)(n * pitch);
                const int64_t x0 = (int64_t)(pair / p.topk) * p.ldx;
                float inv;
                if (DOWN) inv = put_activations<BY16>(L.hidden + (int64_t)pair * p.H, K, nkb, dst, lane);
                else if (p.type == Q4_BF16) inv = put_activations<BY16>(static_cast<const __nv_bfloat16*>(p.X) + x0, K, nkb, dst, lane);
                else inv = put_activations<BY16>(static_cast<const __half*>(p.X) + x0, K, nkb, dst, lane);
                if (lane == 0) inverse[n] = inv;
            }
            sync_consumers();
        }
        float acc[4][NT][4] = {};
        for (int b = (warp - it0) & (CONSUMERS - 1); b < nkb; b += CONSUMERS) {
            const int it = it0 + b, st = it % STAGES;
            mbar_wait_suspend(bar_full(st), (uint32_t)(it / STAGES) & 1u, abort_flag, p.status);
            const uint32_t ws = sbase + st * C::STAGE, sc = scales_s + st * C::SCALE;
            const uint32_t xs = act_s + (uint32_t)(g * pitch + b * SK * 2 + t * 16);
            const int nw = (int)words_of(K, BY16) - b * C::WORDS;      // words that exist
            auto masked = [&](int row, int w) {
                const uint32_t v = (uint32_t)lds32(sc + 4u * (uint32_t)(w * TROWS + row));
                return w < nw - 1 ? v : w == nw - 1 ? v & valid_bytes(K - b * SK - w * word_cols(BY16), group_of(BY16)) : 0u;
            };
            if constexpr (BY16) {
                uint32_t sw[8];
#pragma unroll
                for (int r = 0; r < 8; ++r) sw[r] = masked(8 * r + g, t) & 0x7F7F7F7Fu;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    // 32 codes of each of my rows: piece 2 t + h
                    uint4 c[8];
#pragma unroll
                    for (int r = 0; r < 8; ++r) c[r] = lds128(ws + (uint32_t)((8 * r + g) * SROWB + (((2 * t + h) ^ g) << 4)));
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint4 x[NT];
#pragma unroll
                        for (int j = 0; j < NT; ++j) x[j] = lds128(xs + (uint32_t)(8 * j * pitch + (4 * h + i) * 64));
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            uint32_t a[4], d[4];
                            const uint4 &ca = c[2 * r], &cd = c[2 * r + 1];
                            values8(i == 0 ? ca.x : i == 1 ? ca.y : i == 2 ? ca.z : ca.w, a);
                            values8(i == 0 ? cd.x : i == 1 ? cd.y : i == 2 ? cd.z : cd.w, d);
                            const uint32_t pick = i < 2 ? 0x1010 : 0x3232;
                            const uint32_t sa = __byte_perm(scales2(sw[2 * r] >> (16 * h)), 0, pick);
                            const uint32_t sd = __byte_perm(scales2(sw[2 * r + 1] >> (16 * h)), 0, pick);
#pragma unroll
                            for (int k = 0; k < 4; ++k) { a[k] = mul2(a[k], sa); d[k] = mul2(d[k], sd); }
#pragma unroll
                            for (int j = 0; j < NT; ++j) {
                                mma_f16(acc[r][j], a[0], d[0], a[1], d[1], x[j].x, x[j].y);
                                mma_f16(acc[r][j], a[2], d[2], a[3], d[3], x[j].z, x[j].w);
                            }
                        }
                    }
                }
            } else {
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    uint32_t sw[8];
#pragma unroll
                    for (int r = 0; r < 8; ++r) sw[r] = masked(8 * r + g, w);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint4 x[NT];
#pragma unroll
                        for (int j = 0; j < NT; ++j) x[j] = lds128(xs + (uint32_t)(8 * j * pitch + (4 * w + i) * 64));
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const uint32_t at = ws + (uint32_t)((16 * r + g) * SROWB + (((4 * w + i) ^ g) << 4) + 4 * t);
                            uint32_t a[4], d[4];
                            values8((uint32_t)lds32(at), a);
                            values8((uint32_t)lds32(at + 8 * SROWB), d);
                            // 2^(byte - 127): 0 is 2^-127, 255 becomes NaN
                            auto scale = [&](uint32_t word) {
                                const uint32_t top = i == 0 ? word << 24 : i == 1 ? (word << 16) & 0xFF000000u : i == 2 ? (word << 8) & 0xFF000000u : word & 0xFF000000u;
                                const float s = __uint_as_float(max(top >> 1, 0x00400000u));
                                return fmaf(s, 0.0f, s);
                            };
                            const float sa = scale(sw[2 * r]), sd = scale(sw[2 * r + 1]);
#pragma unroll
                            for (int j = 0; j < NT; ++j) {
                                float m[4] = {};
                                mma_f16(m, a[0], d[0], a[1], d[1], x[j].x, x[j].y);
                                mma_f16(m, a[2], d[2], a[3], d[3], x[j].z, x[j].w);
                                acc[r][j][0] = fmaf(m[0], sa, acc[r][j][0]);
                                acc[r][j][1] = fmaf(m[1], sa, acc[r][j][1]);
                                acc[r][j][2] = fmaf(m[2], sd, acc[r][j][2]);
                                acc[r][j][3] = fmaf(m[3], sd, acc[r][j][3]);
                            }
                        }
                    }
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_empty(st));
        }
        // partial sums [warp][pair][row]
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    sts32(part_s + 4u * (uint32_t)((warp * C::N + 8 * j + 2 * t + (i & 1)) * C::PITCH + 16 * r + 8 * (i >> 1) + g),
                          __float_as_int(acc[r][j][i]));
        sync_consumers();
        auto sum = [&](int n, int row) {
            float v = 0.0f;
#pragma unroll
            for (int k = 0; k < CONSUMERS; ++k) v += __int_as_float(lds32(part_s + 4u * (uint32_t)((k * C::N + n) * C::PITCH + row)));
            return v * inverse[n] * f;
        };
        for (int i = threadIdx.x; i < count * per_tile; i += CONSUMERS * 32) {
            const int n = i / per_tile, row = i % per_tile, pair = order[begin + n];
            if (r0 + row >= rows) continue;
            const float v = sum(n, row);
            if (DOWN) {
                L.y[(int64_t)pair * p.D + r0 + row] = v;
            } else {
                const float s = v / (1.0f + expf(-v));
                L.hidden[(int64_t)pair * p.H + r0 + row] = p.gated ? s * sum(n, BOXROWS + row) : s;
            }
        }
        if (DOWN) {
            __threadfence();
            sync_consumers();                                  // all of the tile is written
            if (threadIdx.x == 0) words[2] = atomicAdd(L.done + r0 / TROWS, 1) == nunits - 1;
        }
        sync_consumers();                                      // partial sums have been read
        if (DOWN && words[2]) {
            // these columns of every pair are there
            __threadfence();
            for (int i = threadIdx.x; i < p.tokens * TROWS; i += CONSUMERS * 32) {
                const int tok = i / TROWS, d = r0 + i % TROWS;
                if (d >= p.D) continue;
                float out = 0.0f;
#pragma unroll 4
                for (int j = 0; j < p.topk; ++j) {
                    const int64_t pair = (int64_t)tok * p.topk + j;
                    if ((unsigned)__ldg(p.ids + pair) >= (unsigned)p.E) continue;
                    out = fmaf(p.w ? __ldg(p.w + pair) : 1.0f, __ldcg(L.y + pair * p.D + d), out);
                }
                store_value(p.Out, tok * p.ldo + d, p.type, out);
            }
        }
    }
    if (DOWN && nunits == 0)                                   // no pair at all
        for (int64_t i = (int64_t)blockIdx.x * CONSUMERS * 32 + threadIdx.x; i < (int64_t)p.tokens * p.D; i += (int64_t)gridDim.x * CONSUMERS * 32)
            store_value(p.Out, i / p.D * p.ldo + i % p.D, p.type, 0.0f);
}

constexpr int SMEM_MOST = 232448;

template <bool BY16, int NT> static int stages_for(int K)
{
    using C = LayerCfg<BY16, NT>;
    const int nkb = (K + SK - 1) / SK;
    return C::bytes(16, nkb) <= SMEM_MOST ? 16 : C::bytes(8, nkb) <= SMEM_MOST ? 8 : 0;
}

template <bool BY16, int NT, bool DOWN>
static cudaError_t launch_layer(LayerLaunch L, const CUtensorMap& m, cudaStream_t st)
{
    using C = LayerCfg<BY16, NT>;
    auto kernel = layer_kernel<BY16, NT, DOWN>;
    static bool ready[64] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!ready[dev]) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_MOST);
        if (e != cudaSuccess) return e;
        ready[dev] = true;
    }
    const int K = DOWN ? L.p.H : L.p.D;
    L.stages = stages_for<BY16, NT>(K);
    return f8::launch(kernel, (unsigned)(2 * f8_pairs_of_device()), LAYER_THREADS, C::bytes(L.stages, (K + SK - 1) / SK), st, m, L);
}

template <bool BY16, int NT>
static cudaError_t launch_both(const LayerLaunch& L, const CUtensorMap& up, const CUtensorMap& down, cudaStream_t st)
{
    const cudaError_t e = launch_layer<BY16, NT, false>(L, up, st);
    return e != cudaSuccess ? e : launch_layer<BY16, NT, true>(L, down, st);
}

}  // namespace f4

using namespace f4;

// The workspace: a counter per tile of output columns, hidden values, what each pair adds to its token.
static int64_t counters_bytes(int32_t D) { return (((int64_t)D + TROWS - 1) / TROWS * 4 + 255) / 256 * 256; }

int64_t expert_layer_f4_ws_bytes(int64_t pairs, int32_t D, int32_t H)
{
    return counters_bytes(D) + 4 * pairs * ((int64_t)H + D);
}

// 16-bit activations whose rows fit shared memory eight at a time, weights that a tensor map can name, few pairs.
bool expert_layer_f4_stream_supported(const f4::LayerParams& p, bool by16)
{
    const int K = p.D > p.H ? p.D : p.H;
    const int64_t rows1 = (int64_t)p.E * (p.gated ? 2 : 1) * p.H, rows2 = (int64_t)p.E * p.D;
    return p.type != Q4_F32 && (int64_t)p.tokens * p.topk <= MAX_PAIRS && K <= 16384 &&
           (by16 ? stages_for<true, 1>(K) : stages_for<false, 1>(K)) > 0 && rows1 < INT32_MAX - 512 && rows2 < INT32_MAX - 512 &&
           (uintptr_t)p.W1 % 16 == 0 && (uintptr_t)p.W2 % 16 == 0 && p.ldw1 % 16 == 0 && p.ldw2 % 16 == 0;
}

q4_status launch_expert_layer_f4_stream(const f4::LayerParams& p, bool by16, cudaStream_t st)
{
    const int64_t pairs = (int64_t)p.tokens * p.topk;
    LayerLaunch L{p, nullptr, nullptr, nullptr, 0};
    L.done = static_cast<int*>(p.ws);
    L.hidden = reinterpret_cast<float*>(static_cast<uint8_t*>(p.ws) + counters_bytes(p.D));
    L.y = L.hidden + pairs * p.H;
    CUtensorMap up, down;
    if (!make_byte_map(&up, p.W1, p.ldw1, p.E * (p.gated ? 2 : 1) * p.H, (p.D + 1) / 2, BOXROWS) ||
        !make_byte_map(&down, p.W2, p.ldw2, p.E * p.D, (p.H + 1) / 2, BOXROWS)) return Q4_ERR_CUDA;
    // sixteen pairs per unit where experts are hit by more than eight on average: the weights pass once for them
    const int K = p.D > p.H ? p.D : p.H;                       // both kernels alike
    const bool two = pairs > 8 * (int64_t)p.E && (by16 ? stages_for<true, 2>(K) : stages_for<false, 2>(K)) > 0;
    cudaError_t e;
    if (by16) e = two ? launch_both<true, 2>(L, up, down, st) : launch_both<true, 1>(L, up, down, st);
    else e = two ? launch_both<false, 2>(L, up, down, st) : launch_both<false, 1>(L, up, down, st);
    return e == cudaSuccess ? Q4_OK : Q4_ERR_CUDA;
}

}  // namespace q4
