// Block-scaled tcgen05 products of e2m1 operands: instruction wrappers and the scales' way into tensor memory,
// shared by the CTA-pair kernel and the few-rows kernel.
//
// An instruction multiplies 64 depth values (32 bytes of codes per row).  Its scales lie in tensor memory: the word of
// row r in lane r % 32 and column r / 32 of a group of four columns per 128 rows, the same in all four lane quarters.
// In shared memory such a group is an atom of 512 bytes, lane by lane, that tcgen05.cp copies to the four quarters.
// BY16 an instruction takes a word's four scales (scale_vec::4X), else two of them (scale_vec::2X), picked by the
// descriptor's scale ids.
#pragma once

#include "q4_f4.cuh"
#include "q4_tc_ptx.cuh"

namespace q4 {

bool make_byte_map(CUtensorMap* tm, const uint8_t* base, int64_t ld, int rows, int kbytes, int box_rows);

namespace f4 {

constexpr int ROWB = 128;                        // bytes of codes per row and stage
constexpr int STAGE_K = 2 * ROWB;                // depth values per stage: four instructions
constexpr int ATOM = 512;                        // bytes of the scales of 128 rows' word
template <bool BY16> constexpr int kWords = BY16 ? 4 : 2;          // words of scales per row and stage

// D = f32, A = B = e2m1, K-major; scales e4m3 (BY16) or powers of two.  `id`: first byte of the word that is used.
template <bool BY16> __host__ __device__ constexpr uint32_t idesc(int m, int n, int id)
{
    return ((uint32_t)id << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | (BY16 ? 0u : 1u << 23) |
           ((uint32_t)(m >> 4) << 24) | ((uint32_t)id << 29);
}

template <bool BY16, int GROUP>
__device__ __forceinline__ void tc_mma_f4(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t id, uint32_t sa, uint32_t sb,
                                          uint32_t accumulate)
{
    if constexpr (BY16 && GROUP == 2)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::2.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], %1, %2, %3, [%5], [%6], p;\n\t}"
                     ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(id), "r"(accumulate), "r"(sa), "r"(sb) : "memory");
    else if constexpr (BY16)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::1.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], %1, %2, %3, [%5], [%6], p;\n\t}"
                     ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(id), "r"(accumulate), "r"(sa), "r"(sb) : "memory");
    else if constexpr (GROUP == 2)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%5], [%6], p;\n\t}"
                     ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(id), "r"(accumulate), "r"(sa), "r"(sb) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%5], [%6], p;\n\t}"
                     ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(id), "r"(accumulate), "r"(sa), "r"(sb) : "memory");
}

// An atom of scales to four columns of tensor memory (of both CTAs of a pair, each from its own shared memory).  In the
// order of the issuing thread's products.
template <int GROUP> __device__ __forceinline__ void tc_copy_scales(uint32_t d_tmem, uint64_t desc)
{
    if constexpr (GROUP == 2)
        asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(d_tmem), "l"(desc) : "memory");
    else
        asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(d_tmem), "l"(desc) : "memory");
}
// Unswizzled rows of 16 bytes, eight of them a piece of 128 bytes, the pieces one behind the other.
__device__ __forceinline__ uint64_t scales_desc(uint32_t saddr)
{
    return (uint64_t)((saddr & 0x3FFFFu) >> 4) | (8ull << 16) | (8ull << 32) | (1ull << 46);
}

// A load that stays where it is written, ahead of its use; 0 where `in` is false.
__device__ __forceinline__ uint32_t load_word(const uint32_t* at, bool in)
{
    uint32_t w;
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %2, 0;\n\tmov.b32 %0, 0;\n\t@p ld.global.nc.b32 %0, [%1];\n\t}"
                 : "=r"(w) : "l"(at), "r"((int)in));
    return w;
}

// Waits for the thread's tensor-memory loads; the loaded registers pass through it, so that nothing that uses them can be
// moved above it.
__device__ __forceinline__ void tc_wait_ld32(uint32_t (&r)[32])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                   "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]),
                   "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]),
                   "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
                 :: "memory");
}

__device__ __forceinline__ void tc_wait_ld16(uint32_t (&r)[16])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                   "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
                 :: "memory");
}

struct Tile {
    int m0, m_end;                   // first row and end of its segment
    int n0;                          // first column
    int64_t brow;                    // its row of Bt
    int e;                           // expert
};

// The walk over tiles of TR rows x TN columns.  Called by whole warps: an expert's segment is found 32 experts at a time.
template <int TR, int TN>
struct Walk {
    const GemmParams& g;
    int tiles_m, tiles_n, lane;
    int e0 = 0, cum = 0, lo = 0, hi = 0, incl = 0;
    __device__ Walk(const GemmParams& g_, int tiles_m_, int tiles_n_, int lane_) : g(g_), tiles_m(tiles_m_), tiles_n(tiles_n_), lane(lane_)
    {
        if (g.E) load();
    }
    __device__ void load()
    {
        const int e = e0 + lane;
        lo = hi = 0;
        if (e < g.E) {
            lo = clamp_to(g.starts[e], 0, g.M);
            hi = clamp_to(g.starts[e + 1], lo, g.M);
        }
        incl = (hi - lo + TR - 1) / TR * tiles_n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int u = __shfl_up_sync(0xFFFFFFFFu, incl, o);
            if (lane >= o) incl += u;
        }
    }
    __device__ bool get(int t, Tile& o)
    {
        if (g.E) {
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
            const int tm = (end - s + TR - 1) / TR;
            const int local = t - cum - before, n = local / tm;        // row tiles fastest: they share the weights
            o.m0 = s + (local - n * tm) * TR;
            o.m_end = end;
            o.n0 = n * TN;
            o.e = e0 + i;
            o.brow = (int64_t)o.e * g.N + o.n0;
            return true;
        }
        if (t >= tiles_m * tiles_n) return false;
        // bands of eight row tiles: the tiles in flight at a time share rows of both operands
        const int band = t / (8 * tiles_n), r = t - band * 8 * tiles_n;
        const int h = min(8, tiles_m - band * 8), n = r / h;
        o.m0 = (band * 8 + r - n * h) * TR;
        o.m_end = g.M;
        o.n0 = n * TN;
        o.e = 0;
        o.brow = o.n0;
        return true;
    }
};

// What brings words of scales to atoms: a team of PARTS warps takes a stage, TEAMS teams in turn, a team's next three stages
// under way.  The wait for a team's stage before told that the stages up to STAGES + TEAMS back are consumed, so the
// parity waited for cannot be that of an older round.  Place: moves to stage (the team's next) and says where this
// warp's words are; false: there is none.
template <int WORDS, bool BY16, int STAGES, int TEAMS, typename Place, typename Put>
__device__ __forceinline__ void bring_scales(int team, int K, uint32_t abort_flag, Place&& place, Put&& put)
{
    const int nw = (int)words_of(K, BY16);
    const uint32_t last_mask = valid_bytes(K - (nw - 1) * word_cols(BY16), group_of(BY16));
    struct Stage { uint4 v[WORDS]; int word0; };
    // (the mask of a matrix's last word is applied when a stage is put: any use of a word at its load would wait for it)
    auto masked = [&](Stage& s) -> const uint4 (&)[WORDS] {
#pragma unroll
        for (int w = 0; w < WORDS; ++w) {
            const uint32_t mask = s.word0 + w == nw - 1 ? last_mask : 0xFFFFFFFFu;
            s.v[w] = make_uint4(s.v[w].x & mask, s.v[w].y & mask, s.v[w].z & mask, s.v[w].w & mask);
        }
        return s.v;
    };
    uint32_t it = (uint32_t)team;
    auto load = [&](Stage& s) {
        const uint32_t* src;
        int64_t ld;
        int rows;                                              // that exist from my lane's first on, 32 apart
        if (!place(src, ld, rows, s.word0)) return false;
#pragma unroll
        for (int w = 0; w < WORDS; ++w) {
            const uint32_t* at = src + (s.word0 + w) * ld;
            const bool in = s.word0 + w < nw;
            s.v[w] = make_uint4(load_word(at, in && rows > 0), load_word(at + 32, in && rows > 32), load_word(at + 64, in && rows > 64),
                                load_word(at + 96, in && rows > 96));
        }
        return true;
    };
    Stage a, b, c;
    bool ha = load(a), hb = load(b), hc = load(c);
    while (ha && !lds32(abort_flag)) {
        put(it, masked(a));
        it += TEAMS;
        ha = load(a);
        if (!hb) break;
        put(it, masked(b));
        it += TEAMS;
        hb = load(b);
        if (!hc) break;
        put(it, masked(c));
        it += TEAMS;
        hc = load(c);
    }
}

}  // namespace f4
}  // namespace q4
