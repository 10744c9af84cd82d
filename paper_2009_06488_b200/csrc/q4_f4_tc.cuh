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

}  // namespace f4
}  // namespace q4
