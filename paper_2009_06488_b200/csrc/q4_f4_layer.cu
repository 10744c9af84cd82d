// Expert layer for a few tokens on e2m1 weights with microscales: two kernels that stream the weights of the experts that
// are hit, once, from HBM through the block-scaled tensor-core product, and a sum.
//
//   kernel 1 (up)     h = silu(G_e x) * (U_e x)  (or silu(G_e x)) of every pair of a token and an expert, binary32
//   kernel 2 (down)   y = W2_e h of every pair, binary32
//   kernel 3 (sum)    Out[t] = sum_j w[t][j] y in the order of j
//
// The tensor core multiplies e2m1 by e2m1, and activations are not quantized: a group of them is written as a sum of PARTS
// e2m1 vectors under one scale 2^a,
//   x = 2^a (c0 + 2^-2 c1 + 2^-5 c2 + 2^-8 c3 + ... + 2^-17 c6) + rest,   max |x| / 2^a in [2, 4),
// the rest at most half a step of the last, 2^-20 of the group's largest value: binary16 and bfloat16 values that are not far
// below it are exact.  x / 2^a is rounded once to an integer of steps 2^-18; c0 is an integer of -4..4 and the others are half
// of its digits to base 8, -4..3: codes 0 to 4 of e2m1 are 0, 1/2, 1, 3/2, 2.  (Parts made one after the other in floating
// point, each the nearest to what is left, took three times the instructions.)
// The parts are rows of the product's second operand and their results are added in binary32.  The scale is
// that of the weights' kind: a power of two per 32, or per 16 one in e4m3 times a power of two for the row.  e4m3 holds 18
// powers of two, so that a group more than 2^17 below the row's largest value has the steps of one that is not: its rest is 2^-37
// of the row's largest.  (20 bits are enough for what the layer writes, 11 at most; binary32 activations run the general kernels.)
//
// Every block sorts the pairs by expert for itself (a few hundred numbers).  A unit is up to NTOK pairs of one expert, a
// tile 128 rows of its weights (gated: 64 of G and the same 64 of U) by PARTS * NTOK columns, the whole depth.  (A product
// of 128 rows takes about 118 clk however few its columns are: with tiles of 64 rows these were the bound.)  One
// persistent block per SM walks tiles, a unit's one after the other:
//
//   warp 0        producer     stages of 256 depth values: two boxes of 64 rows by TMA (128-byte swizzle)
//   warp 1        MMA issuer   a stage's scales to tensor memory, then four products
//   warps 2, 3    scales       a stage each in turn: the rows' words, two turns ahead, put in atoms
//   warps 4..7    epilogue     parts added, gate and product meet through shared memory
//   warps 8..23   activations  the next unit's parts and scales, while this one's are multiplied
//
// Bound: HBM, behind each kernel's start (sorting, the first unit's parts: 7 us of the first) and beside blocks with a tile
// more than others (7 against 6.2 on average).  64 experts of 2048 -> 1024 (gated) -> 2048: sixteen tokens 46 us = 3.6 TB/s of
// weights (50 experts are hit), one token (8 experts) 19 us.  What was tried: the sum in kernel 2 by the block that finishes columns last (its tail
// 6 to 14 us), or by warps of their own that count each token's pairs (16 tokens 47.5 against 46.6 us, one 20.1 against 19.1,
// 32 by 16 68 against 62); all in one cooperative kernel (63); later stages to L2 ahead of their copies (54); codes to
// binary16 in registers and warp-level matrix instructions, the depth spread over a block's warps (86) or a strip of rows per
// warp, brought by 16-byte copies (75) or TMA (77): eight instructions per 16 codes left HBM at a third of its rate.
#include <cuda.h>

#include "q4_f4_tc.cuh"

namespace q4 {
namespace f4 {

constexpr int PARTS = 7;
constexpr int TROWS = 128, BOXROWS = 64;          // weights' rows of a tile and of a copy
constexpr int MAX_PAIRS = 1024;                  // sorted by each block
constexpr int ACT0 = 8, ACTS = 16;               // first of the activations' warps, their number
static_assert(ACTS * 32 == 512, "the activations' warps meet");
constexpr int LAYER_THREADS = (ACT0 + ACTS) * 32;
constexpr int MAX_STAGES = 12;

// Shared memory, in this order: stages of codes, their atoms, units' parts, their atoms, lists and the rest.
template <bool BY16, int NTOK> struct LayerCfg {
    static constexpr int WORDS = kWords<BY16>;
    static constexpr int N = 8 * NTOK;                         // columns of a tile (PARTS * NTOK, a multiple of 16)
    static constexpr int STAGE = TROWS * ROWB, ATOMS = WORDS * ATOM;
    static constexpr int BLOCK = N * ROWB + ATOMS;             // parts of 256 depth values, and their scales
    static constexpr int LISTS = MAX_PAIRS * 2 * 4 + (Q4_MAX_EXPERTS + 32) * 4 * 2;
    static constexpr int REST = 4 * 8 * 4 + 8 * 4 + BOXROWS * NTOK * 4 + (2 * MAX_STAGES + 8) * 8 + 8;
    static constexpr int COL_SCALE = 2 * N;                    // tensor memory: two accumulators, two buffers of scales
    static constexpr int COLS = 256;
    static_assert(PARTS * NTOK <= N && COL_SCALE + 2 * 2 * WORDS * 4 <= COLS, "tensor memory");
    static __host__ __device__ constexpr int bytes(int stages, int bufs, int nkb)
    {
        return stages * (STAGE + ATOMS) + bufs * nkb * BLOCK + LISTS + REST + 1024;
    }
};

struct LayerLaunch {
    LayerParams p;
    float* hidden;                   // [pairs][H]
    float* y;                        // [pairs][D]
    int stages, bufs;
};

// Sorts the pairs by expert: order[] = pairs, expert by expert, in their own order; units of up to N pairs.  All threads.
template <int N, int THREADS>
__device__ __forceinline__ int sort_pairs(const LayerParams& p, uint16_t* order, uint16_t* rank, uint16_t* unit, int* first, int* units)
{
    const int n = p.tokens * p.topk, lane = threadIdx.x & 31, padded = (p.E + 31) & ~31;
    uint16_t* const expert = unit + MAX_PAIRS;                 // of each pair
    for (int i = threadIdx.x; i < n; i += THREADS) {
        const unsigned e = (unsigned)__ldg(p.ids + i);
        expert[i] = (uint16_t)(e < (unsigned)p.E ? e : 0xFFFFu);
    }
    for (int e = threadIdx.x; e < padded; e += THREADS) first[e] = 0;
    __syncthreads();
    if (threadIdx.x < 32) {
        for (int i0 = 0; i0 < n; i0 += 32) {
            const int i = i0 + lane, e = i < n ? expert[i] : 0xFFFF;
            const bool in = e != 0xFFFF;
            const unsigned same = __match_any_sync(0xFFFFFFFFu, e), before = same & ((1u << lane) - 1u);
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
            const int c = first[e0 + lane], both = c | ((c + N - 1) / N) << 16;      // at most 1024 of either
            int sum = both;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int a = __shfl_up_sync(0xFFFFFFFFu, sum, o);
                if (lane >= o) sum += a;
            }
            first[e0 + lane] = at + (sum & 0xFFFF) - c;
            units[e0 + lane] = un + (sum >> 16) - (both >> 16);
            sum = __shfl_sync(0xFFFFFFFFu, sum, 31);
            at += sum & 0xFFFF;
            un += sum >> 16;
        }
        if (lane == 0) {
            first[padded] = at;
            units[padded] = un;
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += THREADS) {
        const int e = expert[i];
        if (e != 0xFFFF) order[first[e] + rank[i]] = (uint16_t)i;
    }
    for (int e = threadIdx.x; e < p.E; e += THREADS)
        for (int u = units[e]; u < units[e + 1]; ++u) unit[u] = (uint16_t)e;
    __syncthreads();
    return units[padded];
}


// 8 consecutive values from k on, 0 where there are none.
template <typename T> __device__ __forceinline__ f8::Eight<T> eight_at(const T* row, int k, int K)
{
    f8::Eight<T> e;
    if ((uintptr_t)row % 16 == 0 && k + 8 <= K) {
#pragma unroll
        for (int q = 0; q < f8::Eight<T>::NW / 4; ++q) {
            const uint4 u = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint8_t*>(row + k) + 16 * q);
            e.w[4 * q] = u.x; e.w[4 * q + 1] = u.y; e.w[4 * q + 2] = u.z; e.w[4 * q + 3] = u.w;
        }
    } else {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = f8::to_f(row[min(k + i, K - 1)]);      // (without conditions: all under way together)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = k + i < K ? v[i] : 0.0f;
        f8::pack8(e, v);
    }
    return e;
}
template <typename T> __device__ __forceinline__ uint32_t largest(const f8::Eight<T>& e)
{
    uint32_t a = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) a = max(a, __float_as_uint(e.get(i)) & 0x7FFFFFFFu);
    return a;
}

// The field at bit `at` of eight values' halves of words, value n to nibble n.
__device__ __forceinline__ uint32_t nibbles(const uint32_t (&w)[4], int at, uint32_t field)
{
    uint32_t r = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) r |= (4 * j >= at ? w[j] << (4 * j - at) : w[j] >> (at - 4 * j)) & (field | field << 16) << (4 * j);
    return r;
}
// Nibbles 0..7 that stand for digits -4..3 to the codes of half of these (the code of d / 2 is |d| and the sign).
__device__ __forceinline__ uint32_t digit_codes(uint32_t w)
{
    const uint32_t neg = (~w & 0x44444444u) >> 2;
    return ((w ^ neg * 3u) & 0x33333333u) + neg * 9u;          // negative: 8 + (~d & 3) + 1
}

// Parts and scales of 256 values of a pair (column n of the unit), eight per lane, by a warp.  rowe: the biased exponent of
// the row's factor (BY16).  parts, atoms: the block's places.
template <bool BY16, int NTOK, typename T>
__device__ __forceinline__ void put_parts(const f8::Eight<T>& v, int n, uint32_t rowe, uint32_t parts, uint32_t atoms, int lane)
{
    uint32_t a = largest(v);
    a = max(a, __shfl_xor_sync(0xFFFFFFFFu, a, 1));
    if (!BY16) a = max(a, __shfl_xor_sync(0xFFFFFFFFu, a, 2));
    const int e = (int)(a >> 23);
    uint32_t byte;
    int s;                                                     // biased exponent of the scale
    if (BY16) {
        const int se = clamp_to(e - 1 - (int)rowe, -9, 8);     // of its e4m3 part
        byte = e == 255 ? 0x7Fu : se >= -6 ? (uint32_t)(se + 7) << 3 : 1u << (se + 9);
        s = se + (int)rowe;
    } else {
        s = max(e, 2) - 1;
        byte = e == 255 ? 255u : (uint32_t)s;
    }
    const float inv = __uint_as_float((uint32_t)(254 - s) << 23);
    // x / 2^a in steps of 2^-18, plus 4 in each digit to base 8 (as digits of -4..3 are asked for) and in what is above them
    uint32_t y[8], lo[4], hi[4];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = __float_as_uint(fmaf(v.get(i) * inv, 262144.0f, 12582912.0f)) + (0x124924u - 0x4B400000u);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        lo[j] = __byte_perm(y[j], y[j + 4], 0x5410);           // bits 0..15 of both
        hi[j] = __byte_perm(y[j], y[j + 4], 0x6521);           // bits 8..23
    }
    auto put = [&](int q, uint32_t codes) {
        const int row = q * NTOK + n;
        sts32(parts + (uint32_t)(row * ROWB) + (uint32_t)((((lane >> 2) ^ row) & 7) << 4) + (uint32_t)(lane & 3) * 4u, (int)codes);
    };
    {
        // 0..8 for -4..4, whose codes are 0, 2, 4, 5, 6 and the sign: bit by bit, eight values at a time
        constexpr uint32_t ONES = 0x11111111u;
        const uint32_t w = nibbles(hi, 10, 0xFu), b0 = w, b1 = w >> 1, b2 = w >> 2, b3 = w >> 3, neg = ~(b2 | b3);
        const uint32_t c2 = (neg & ~(b1 & b0)) | (~neg & (b3 | b1)), c1 = (neg & ~(b1 ^ b0)) | (~neg & (b3 | (~b1 & b0))),
                       c0 = b0 & (b1 ^ neg);
        put(0, (c0 & ONES) | (c1 & ONES) << 1 | (c2 & ONES) << 2 | (neg & ONES) << 3);
    }
    put(1, digit_codes(nibbles(hi, 7, 7u)));
#pragma unroll
    for (int q = 2; q < PARTS; ++q) put(q, digit_codes(nibbles(lo, 3 * (PARTS - 1 - q), 7u)));
    // the words: by 16 a word is 8 lanes' (a group two), else 16 lanes' (a group four)
    constexpr int G = BY16 ? 2 : 4;
    uint32_t w = byte << (8 * (lane / G & 3));
    w |= __shfl_xor_sync(0xFFFFFFFFu, w, G);
    w |= __shfl_xor_sync(0xFFFFFFFFu, w, 2 * G);
    const int q = lane & (4 * G - 1), row = q * NTOK + n;      // lane q of a word writes it for part q
    if (q < PARTS) sts32(atoms + (uint32_t)(lane / (4 * G) * ATOM + (row & 31) * 16 + (row >> 5) * 4), (int)w);
}

template <bool BY16, int NTOK, bool DOWN>
__global__ void __launch_bounds__(LAYER_THREADS, 1)
layer_kernel(const __grid_constant__ CUtensorMap tmW, const LayerLaunch L)
{
    using C = LayerCfg<BY16, NTOK>;
    const LayerParams& p = L.p;
    extern __shared__ uint8_t smem_raw[];
    const int K = DOWN ? p.H : p.D, nkb = (K + STAGE_K - 1) / STAGE_K, STAGES = L.stages;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t sbase = (smem_u32(smem_raw) + 1023u) & ~1023u, act_s = sbase + STAGES * C::STAGE,
                   atoms_s = act_s + L.bufs * nkb * C::N * ROWB, act_atoms = atoms_s + STAGES * C::ATOMS,
                   lists_s = act_atoms + L.bufs * nkb * C::ATOMS;
    uint8_t* const lists = smem_raw + (lists_s - smem_u32(smem_raw));
    int* const first = reinterpret_cast<int*>(lists);                       // pairs before each expert [E, a multiple of 32, + 1]
    int* const units = first + Q4_MAX_EXPERTS + 32;                         // units before each expert
    uint16_t* const order = reinterpret_cast<uint16_t*>(units + Q4_MAX_EXPERTS + 32);
    uint16_t* const rank = order + MAX_PAIRS;
    uint16_t* const unit = rank + MAX_PAIRS;                                // expert of each unit
    float* const row_factor = reinterpret_cast<float*>(lists + C::LISTS);   // [unit & 3][8]
    unsigned* const row_max = reinterpret_cast<unsigned*>(row_factor + 32); // [8]
    float* const exchange = reinterpret_cast<float*>(row_max + 8);          // [NTOK][BOXROWS]
    const uint32_t bar0 = lists_s + C::LISTS + 4 * 8 * 4 + 8 * 4 + BOXROWS * NTOK * 4;
    auto bar_full   = [&](uint32_t s) { return bar0 + 8u * s; };
    auto bar_empty  = [&](uint32_t s) { return bar0 + 8u * (MAX_STAGES + s); };
    auto bar_tfull  = [&](uint32_t a) { return bar0 + 8u * (2 * MAX_STAGES + a); };
    auto bar_tempty = [&](uint32_t a) { return bar0 + 8u * (2 * MAX_STAGES + 2 + a); };
    auto bar_act    = [&](uint32_t b) { return bar0 + 8u * (2 * MAX_STAGES + 4 + b); };     // a unit's parts are there
    auto bar_used   = [&](uint32_t b) { return bar0 + 8u * (2 * MAX_STAGES + 6 + b); };     // ... and have been multiplied
    const uint32_t abort_flag = bar0 + 8u * (2 * MAX_STAGES + 8), tmem_slot = abort_flag + 4;

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(bar_full(s), 2);       // the copies' announcement, the scales' warp
            mbar_init(bar_empty(s), 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(bar_tfull(a), 1);
            mbar_init(bar_tempty(a), 4);     // the epilogue's warps
            mbar_init(bar_act(a), ACTS);
            mbar_init(bar_used(a), 1);
        }
        sts32(abort_flag, 0);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async_smem();
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tmem_slot), "r"((uint32_t)C::COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    // Kernel 2 starts when every block of kernel 1 has waited for what came before them: what it reads but for the
    // hidden values is there, and its bounded waits ahead of those last as long as kernel 1 at most.
    if (!DOWN) f8::wait_for_predecessor();
    tc_fence_before();
    const int nunits = sort_pairs<NTOK, LAYER_THREADS>(p, order, rank, unit, first, units);
    tc_fence_after();
    const uint32_t tmem_base = (uint32_t)lds32(tmem_slot);
    const bool gated = !DOWN && p.gated;
    const int rows = DOWN ? p.D : p.H;                          // of the output
    const int per = gated ? BOXROWS : TROWS;                    // of them in a tile
    const int each = (rows + per - 1) / per, ntiles = nunits * each;
    const int expert_rows = DOWN ? p.D : gated ? 2 * p.H : p.H, half = gated ? p.H : BOXROWS;
    // a block's tiles lie together
    const int t0 = (int)((int64_t)ntiles * blockIdx.x / gridDim.x), t1 = (int)((int64_t)ntiles * (blockIdx.x + 1) / gridDim.x);

    if (warp == 0) {
        // ------------------------------------------------------------ producer
        uint32_t st = 0, ph = 0;
        for (int tile = t0; tile < t1 && !lds32(abort_flag); ++tile) {
            const int u = tile / each, row = unit[u] * expert_rows + (tile - u * each) * per;
            for (int b = 0; b < nkb; ++b) {
                mbar_wait(bar_empty(st), ph ^ 1u, abort_flag, p.status);
                if (elect_one()) {
                    const uint32_t dst = sbase + st * C::STAGE;
                    mbar_expect_tx(bar_full(st), (uint32_t)C::STAGE);
                    tma_load_2d(dst, &tmW, b * ROWB, row, bar_full(st));
                    tma_load_2d(dst + BOXROWS * ROWB, &tmW, b * ROWB, row + half, bar_full(st));
                }
                __syncwarp();
                if (++st == (uint32_t)STAGES) { st = 0; ph ^= 1u; }
            }
        }
        settle(abort_flag);
    } else if (warp == 1) {
        // ------------------------------------------------------------ MMA issuer
        const uint64_t desc0 = make_kmajor_sw128_desc(sbase), act0 = make_kmajor_sw128_desc(act_s), scales0 = scales_desc(atoms_s),
                       act_scales0 = scales_desc(act_atoms);
        uint32_t st = 0, ph = 0, buf = 0, acc = 0, aph = 0, ab = 0, abph = 0;
        int at_unit = t0 < t1 ? t0 / each : 0;
        if (t0 < t1) mbar_wait_suspend(bar_act(0), 0, abort_flag, p.status);
        for (int tile = t0; tile < t1 && !lds32(abort_flag); ++tile) {
            const int u = tile / each;
            if (u != at_unit) {
                at_unit = u;
                if (++ab == (uint32_t)L.bufs) { ab = 0; abph ^= 1u; }
                mbar_wait_suspend(bar_act(ab), abph, abort_flag, p.status);
            }
            const bool unit_follows = tile + 1 < t1 && (tile + 1) / each != u;
            mbar_wait(bar_tempty(acc), aph ^ 1u, abort_flag, p.status);
            for (int b = 0; b < nkb; ++b) {
                mbar_wait(bar_full(st), ph, abort_flag, p.status);
                tc_fence_after();
                if (elect_one()) {
                    const uint64_t adesc = desc0 + (uint64_t)(st * (uint32_t)(C::STAGE >> 4));
                    const uint64_t bdesc = act0 + (uint64_t)((ab * nkb + b) * (uint32_t)(C::N * ROWB >> 4));
                    const uint64_t sa_desc = scales0 + (uint64_t)(st * (uint32_t)(C::ATOMS >> 4));
                    const uint64_t sb_desc = act_scales0 + (uint64_t)((ab * nkb + b) * (uint32_t)(C::ATOMS >> 4));
                    const uint32_t sa = tmem_base + C::COL_SCALE + buf * (8 * C::WORDS), sb = sa + 4 * C::WORDS;
#pragma unroll
                    for (int w = 0; w < C::WORDS; ++w) {
                        tc_copy_scales<1>(sa + 4 * w, sa_desc + (uint64_t)(w * (ATOM >> 4)));
                        tc_copy_scales<1>(sb + 4 * w, sb_desc + (uint64_t)(w * (ATOM >> 4)));
                    }
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int w = BY16 ? k : k >> 1;
                        tc_mma_f4<BY16, 1>(tmem_base + acc * C::N, adesc + 2 * k, bdesc + 2 * k, idesc<BY16>(128, C::N, BY16 ? 0 : 2 * (k & 1)),
                                           sa + 4 * w, sb + 4 * w, b | k ? 1u : 0u);
                    }
                    tc_commit(bar_empty(st));
                    if (b == nkb - 1) {
                        if (unit_follows) tc_commit(bar_used(ab));
                        tc_commit(bar_tfull(acc));         // the block's last arrival: it is waited for
                    }
                }
                __syncwarp();
                buf ^= 1u;
                if (++st == (uint32_t)STAGES) { st = 0; ph ^= 1u; }
            }
            aph ^= acc;
            acc ^= 1u;
        }
        settle(abort_flag);
    } else if (warp < 4) {
        // ------------------------------------------------------------ scales
        // (the wait for the stage before told that stages up to STAGES + 2 back are consumed: a parity cannot be an older round's)
        const uint32_t* const S = DOWN ? p.S2 : p.S1;
        const int64_t lds = DOWN ? p.lds2 : p.lds1;
        const int nw = (int)words_of(K, BY16);
        const uint32_t last_mask = valid_bytes(K - (nw - 1) * word_cols(BY16), group_of(BY16));
        int tile = t0, b = warp - 2;                           // what is loaded next
        const uint32_t* at[4] = {};
        auto place = [&]() {
            while (tile < t1 && b >= nkb) {
                b -= nkb;
                ++tile;
            }
            if (tile >= t1) return;
            const int u = tile / each, r0 = (tile - u * each) * per;
            const uint32_t* const base = S + unit[u] * expert_rows;
            // (a row past the end is the last one again: its results are not written)
#pragma unroll
            for (int c = 0; c < 4; ++c)
                at[c] = base + (gated ? min(r0 + 32 * (c & 1) + lane, rows - 1) + (c >> 1) * half : min(r0 + 32 * c + lane, rows - 1));
        };
        auto load = [&](uint4 (&v)[C::WORDS]) {
            if (tile >= t1) return false;
#pragma unroll
            for (int w = 0; w < C::WORDS; ++w) {
                const int word = b * C::WORDS + w;
                const int64_t off = word * lds;
                v[w] = make_uint4(load_word(at[0] + off, word < nw), load_word(at[1] + off, word < nw), load_word(at[2] + off, word < nw),
                                  load_word(at[3] + off, word < nw));
            }
            if ((b += 2) >= nkb) place();
            return true;
        };
        uint32_t it = (uint32_t)(warp - 2);
        int kb = warp - 2;
        auto put = [&](uint4 (&v)[C::WORDS]) {
            while (kb >= nkb) kb -= nkb;
            const uint32_t st = it % (uint32_t)STAGES, ph = it / (uint32_t)STAGES & 1u;
            mbar_wait_suspend(bar_empty(st), ph ^ 1u, abort_flag, p.status);
            const uint32_t dst = atoms_s + st * C::ATOMS + (uint32_t)lane * 16u;
#pragma unroll
            for (int w = 0; w < C::WORDS; ++w) {
                const uint32_t mask = kb * C::WORDS + w == nw - 1 ? last_mask : 0xFFFFFFFFu;
                sts128(dst + (uint32_t)(w * ATOM), make_uint4(v[w].x & mask, v[w].y & mask, v[w].z & mask, v[w].w & mask));
            }
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_full(st));
            it += 2;
            kb += 2;
        };
        place();
        uint4 v0[C::WORDS], v1[C::WORDS];
        bool h0 = load(v0), h1 = load(v1);
        while (h0 && !lds32(abort_flag)) {
            put(v0);
            h0 = load(v0);
            if (!h1) break;
            put(v1);
            h1 = load(v1);
        }
    } else if (warp < 8) {
        // ------------------------------------------------------------ epilogue
        const int h = warp - 4;
        uint32_t acc = 0, aph = 0;
        for (int tile = t0; tile < t1; ++tile) {               // (no way out: the warps meet)
            const int u = tile / each, r0 = (tile - u * each) * per, e = unit[u];
            const int begin = first[e] + (u - units[e]) * NTOK, count = min(NTOK, first[e + 1] - begin);
            const float* const F = DOWN ? p.F2 : p.F1;
            const float f = F ? __ldg(F + e) : 1.0f;
            mbar_wait_suspend(bar_tfull(acc), aph, abort_flag, p.status);
            tc_fence_after();
            const uint32_t ta = tmem_base + ((uint32_t)(h * 32) << 16) + acc * C::N;
            float v[NTOK];
#pragma unroll
            for (int n = 0; n < NTOK; ++n) v[n] = 0.0f;
            // smallest parts first
#pragma unroll
            for (int c = C::N / 32 - 1; c >= 0; --c) {
                uint32_t r[32];
                tc_ld32(ta + 32 * c, r);
                tc_wait_ld32(r);
#pragma unroll
                for (int i = 31; i >= 0; --i) {
                    const int q = (32 * c + i) / NTOK;
                    if (q < PARTS) v[i % NTOK] = fmaf(__uint_as_float(r[i]), q ? 1.0f / (float)(1 << (3 * q - 1)) : 1.0f, v[i % NTOK]);
                }
            }
            // (the rows' factors are read ahead of the arrival: it is what lets their slot be written again)
#pragma unroll
            for (int n = 0; n < NTOK; ++n) v[n] *= (BY16 ? row_factor[(u & 3) * 8 + n] : 1.0f) * f;
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_tempty(acc));
            aph ^= acc;
            acc ^= 1u;
            if (gated) {
                const int r = 32 * (h & 1) + lane;
                if (h >= 2) {
#pragma unroll
                    for (int n = 0; n < NTOK; ++n) exchange[n * BOXROWS + r] = v[n];
                }
                asm volatile("bar.sync 2, 128;" ::: "memory");
                if (h < 2 && r0 + r < rows) {
#pragma unroll
                    for (int n = 0; n < NTOK; ++n)
                        if (n < count) L.hidden[(int64_t)order[begin + n] * p.H + r0 + r] = v[n] / (1.0f + expf(-v[n])) * exchange[n * BOXROWS + r];
                }
                asm volatile("bar.sync 2, 128;" ::: "memory");
            } else {
                const int r = r0 + 32 * h + lane;
                if (r < rows) {
#pragma unroll
                    for (int n = 0; n < NTOK; ++n)
                        if (n < count) {
                            const int pair = order[begin + n];
                            if (DOWN) L.y[(int64_t)pair * p.D + r] = v[n];
                            else L.hidden[(int64_t)pair * p.H + r] = v[n] / (1.0f + expf(-v[n]));
                        }
                }
            }
        }
    } else {
        // ------------------------------------------------------------ activations
        if (DOWN) f8::wait_for_predecessor();                  // the hidden values
        const int me = warp - ACT0;
        const int u0 = t0 < t1 ? t0 / each : 0, u1 = t0 < t1 ? (t1 - 1) / each : -1;
        auto all = [&](auto zero, const void* src, int64_t ld, int div) {
            using T = decltype(zero);
            uint32_t ab = 0, abph = 0;
            for (int u = u0; u <= u1; ++u) {                    // (no way out: the warps meet)
                const int e = unit[u], begin = first[e] + (u - units[e]) * NTOK, count = min(NTOK, first[e + 1] - begin);
                // 256 values of a pair each: pair n, block b; every ACTS-th from mine on
                const int dn = ACTS % count, db = ACTS / count, n0 = me % count, b0 = me / count;
                auto value = [&](int n, int b) {
                    return eight_at(static_cast<const T*>(src) + (int64_t)(order[begin + n] / div) * ld, b * STAGE_K + lane * 8, K);
                };
                auto step = [&](int& n, int& b) {
                    n += dn;
                    b += db;
                    if (n >= count) {
                        n -= count;
                        ++b;
                    }
                };
                f8::Eight<T> v;
                if (b0 < nkb) v = value(n0, b0);
                if (BY16) {
                    // the rows' largest values
                    if (me == 0 && lane < 8) row_max[lane] = 0;
                    asm volatile("bar.sync 3, 512;" ::: "memory");
                    f8::Eight<T> w = v;
#pragma unroll 1
                    for (int n = n0, b = b0; b < nkb;) {
                        const uint32_t a = __reduce_max_sync(0xFFFFFFFFu, largest(w));
                        if (lane == 0) atomicMax(row_max + n, a);
                        step(n, b);
                        if (b < nkb) w = value(n, b);
                    }
                    asm volatile("bar.sync 3, 512;" ::: "memory");
                }
                // biased exponent of a row's factor: its largest group's scale is e4m3's 2^8
                auto row_exponent = [&](int n) {
                    const uint32_t m = row_max[n];
                    return (m >= 0x7F800000u ? 127u : max(m >> 23, 20u)) - 9u;
                };
                mbar_wait_suspend(bar_used(ab), abph ^ 1u, abort_flag, p.status);
                // The slot's last reader is unit u - 4.  This wait tells that unit u - 2 is multiplied (one buffer: u - 1), and its
                // first product waited until the tile two before it, u - 4's or a later one, was read.
                if (BY16 && me == 0 && lane < count) row_factor[(u & 3) * 8 + lane] = __uint_as_float(row_exponent(lane) << 23);
#pragma unroll 1
                for (int n = n0, b = b0; b < nkb;) {
                    const int row = n, at = ab * nkb + b;
                    const f8::Eight<T> now = v;
                    step(n, b);
                    if (b < nkb) v = value(n, b);
                    put_parts<BY16, NTOK>(now, row, BY16 ? row_exponent(row) : 0u, act_s + (uint32_t)(at * C::N * ROWB),
                                          act_atoms + (uint32_t)(at * C::ATOMS), lane);
                }
                fence_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar_act(ab));
                if (BY16) asm volatile("bar.sync 3, 512;" ::: "memory");       // row_max has been read
                if (++ab == (uint32_t)L.bufs) { ab = 0; abph ^= 1u; }
            }
        };
        if (DOWN) all(0.0f, L.hidden, p.H, 1);
        else if (p.type == Q4_BF16) all(__nv_bfloat16(), p.X, p.ldx, p.topk);
        else all(__half(), p.X, p.ldx, p.topk);
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)C::COLS) : "memory");
}

// Out[t][d] = sum_j w[t][j] y of pair (t, j) in the order of j: a thread per value, its eight next terms under way together
// (every address exists; what does not count is left out).
constexpr int SUM_THREADS = 128;
__global__ void __launch_bounds__(SUM_THREADS)
layer_sum_kernel(const LayerLaunch L)
{
    const LayerParams& p = L.p;
    f8::wait_for_predecessor();
    const int per = (p.D + SUM_THREADS - 1) / SUM_THREADS, tok = (int)blockIdx.x / per, d = ((int)blockIdx.x - tok * per) * SUM_THREADS + (int)threadIdx.x;
    if (d >= p.D) return;
    const float* const y = L.y + (int64_t)tok * p.topk * p.D + d;
    float out = 0.0f;
    for (int j0 = 0; j0 < p.topk; j0 += 8) {
        float yv[8], wt[8];
        int id[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int at = min(j0 + j, p.topk - 1);
            id[j] = __ldg(p.ids + tok * p.topk + at);
            wt[j] = p.w ? __ldg(p.w + tok * p.topk + at) : 1.0f;
            yv[j] = __ldcg(y + (int64_t)at * p.D);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j0 + j < p.topk && (unsigned)id[j] < (unsigned)p.E) out = fmaf(wt[j], yv[j], out);
    }
    store_value(p.Out, (int64_t)tok * p.ldo + d, p.type, out);
}

constexpr int SMEM_MOST = 232448;

// Stages and units whose parts are held: two where four stages fit beside them, else one; {0, 0}: none.  Two stages are enough
// to be worth it: eight tokens, 32 experts of 7168 -> 2048 -> 7168 by 16, 169 us = 3.5 TB/s.
struct Room { int stages, bufs; };
template <bool BY16, int NTOK> static Room room_for(int K)
{
    using C = LayerCfg<BY16, NTOK>;
    const int nkb = (K + STAGE_K - 1) / STAGE_K;
    for (int bufs = 2; bufs >= 1; --bufs) {
        int stages = (SMEM_MOST - C::bytes(0, bufs, nkb)) / (C::STAGE + C::ATOMS);
        if (stages > MAX_STAGES) stages = MAX_STAGES;
        if (stages >= (bufs == 2 ? 4 : NTOK == 8 ? 3 : 2)) return {stages, bufs};
    }
    return {0, 0};
}

template <bool BY16, int NTOK, bool DOWN>
static q4_status launch_layer(LayerLaunch L, cudaStream_t st)
{
    using C = LayerCfg<BY16, NTOK>;
    const LayerParams& p = L.p;
    auto kernel = layer_kernel<BY16, NTOK, DOWN>;
    static bool ready[64] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return Q4_ERR_CUDA;
    if (!ready[dev]) {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_MOST) != cudaSuccess) return Q4_ERR_CUDA;
        ready[dev] = true;
    }
    const int K = DOWN ? p.H : p.D;
    const Room r = room_for<BY16, NTOK>(K);
    L.stages = r.stages;
    L.bufs = r.bufs;
    CUtensorMap m;
    if (!make_byte_map(&m, DOWN ? p.W2 : p.W1, DOWN ? p.ldw2 : p.ldw1, p.E * (DOWN ? p.D : p.gated ? 2 * p.H : p.H), (K + 1) / 2, BOXROWS))
        return Q4_ERR_CUDA;
    const int smem = C::bytes(r.stages, r.bufs, (K + STAGE_K - 1) / STAGE_K);
    return f8::launch(kernel, (unsigned)(2 * f8_pairs_of_device()), LAYER_THREADS, smem, st, m, L) == cudaSuccess ? Q4_OK : Q4_ERR_CUDA;
}
template <bool BY16, int NTOK>
static q4_status launch_both(const LayerLaunch& L, cudaStream_t st)
{
    q4_status e = launch_layer<BY16, NTOK, false>(L, st);
    if (e == Q4_OK) e = launch_layer<BY16, NTOK, true>(L, st);
    if (e != Q4_OK) return e;
    const unsigned blocks = (unsigned)(L.p.tokens * ((L.p.D + SUM_THREADS - 1) / SUM_THREADS));
    return f8::launch(layer_sum_kernel, blocks, SUM_THREADS, 0, st, L) == cudaSuccess ? Q4_OK : Q4_ERR_CUDA;
}

}  // namespace f4

using namespace f4;

// The workspace: hidden values, each pair's results.
int64_t expert_layer_f4_ws_bytes(int64_t pairs, int32_t D, int32_t H)
{
    return 4 * pairs * ((int64_t)H + D);
}

template <int NTOK> static bool fits(const f4::LayerParams& p, bool by16)
{
    const int K = p.D > p.H ? p.D : p.H;
    return K <= 16384 && (by16 ? room_for<true, NTOK>(K) : room_for<false, NTOK>(K)).stages > 0;
}

// 16-bit activations whose parts fit shared memory four pairs at a time, weights that a tensor map can name, few pairs.
bool expert_layer_f4_stream_supported(const f4::LayerParams& p, bool by16)
{
    const int64_t rows1 = (int64_t)p.E * (p.gated ? 2 : 1) * p.H, rows2 = (int64_t)p.E * p.D;
    return p.type != Q4_F32 && (int64_t)p.tokens * p.topk <= MAX_PAIRS && fits<4>(p, by16) &&
           rows1 < INT32_MAX - 512 && rows2 < INT32_MAX - 512 &&
           (uintptr_t)p.W1 % 16 == 0 && (uintptr_t)p.W2 % 16 == 0 && p.ldw1 % 16 == 0 && p.ldw2 % 16 == 0;
}

q4_status launch_expert_layer_f4_stream(const f4::LayerParams& p, bool by16, cudaStream_t st)
{
    const int64_t pairs = (int64_t)p.tokens * p.topk;
    LayerLaunch L{p, static_cast<float*>(p.ws), nullptr, 0, 0};
    L.y = L.hidden + pairs * p.H;
    // Eight pairs per unit where their parts fit, so that an expert's weights pass once for them; four where experts are hit by
    // three at most on average: their parts leave room for more stages.
    if (pairs > 3 * (int64_t)p.E && fits<8>(p, by16)) return by16 ? launch_both<true, 8>(L, st) : launch_both<false, 8>(L, st);
    return by16 ? launch_both<true, 4>(L, st) : launch_both<false, 4>(L, st);
}

}  // namespace q4
