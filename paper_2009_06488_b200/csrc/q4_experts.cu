// The expert layer around the experts' products: tokens sorted by expert, rows gathered in that
// order, and the weighted sum back to token order with its gradient.
//
// Sort: a counting sort of n = tokens * topk expert numbers that keeps pairs of one expert in their
// order.  Every warp owns a contiguous piece of the pairs and walks it 32 pairs at a time; a pair's place among its
// block's pairs is the block's pairs of earlier experts + the expert's pairs of earlier warps and rounds + the
// number of lower lanes with the same expert (ballots).  Its row adds the expert's first row (segments rounded up
// to `align`) and the expert's pairs in the chunks of earlier blocks (counted by a first kernel).  Rows are written
// from the block's order, in runs.  All counts are integers: the result does not depend on any order of execution.
// Bound: up to kOneBlock pairs, latency (one block, one launch).  524288 pairs, 11.4 us for a floor of 1: issue and latency
// in turn: the second kernel has 1300 instructions per warp of 128 pairs, issued 56 % of its 9 us, and waits for the
// first kernel's counts; the first (100 per warp) is a trip through memory.
//
// Rows: a row's D values are spread over up to 256 threads, 8 (16 bytes of a 16-bit type) each; a token's
// topk rows are loaded before they are summed, in order and in binary32.  Bound: HBM; issue for rows that do not begin on
// multiples of 16 bytes, which are read and written in aligned pieces (q4_f8.cuh).
#include <type_traits>

#include "q4_f8.cuh"

namespace q4 {
namespace experts {

constexpr int NW = 32;                     // warps of a sort block
constexpr int KEEP = 4;                    // ids a lane keeps in registers (a block of kOneBlock pairs)
constexpr int64_t kOneBlock = 4096;        // pairs per block; up to as many are placed by one block
// More pairs make the chunks larger, not more (every block reads all chunks' counts).  From kMaxChunks * kOneBlock on a
// block's ids no longer fit its registers and its rows go out one by one: 524288 pairs 11.4 us, 524289 13.4, 786432 17.4,
// 1048576 19.3, 2097152 32.
constexpr int kMaxChunks = 128;
constexpr int64_t kRowsPerBlock = 2048;    // rows without a pair per further block

static int chunks_of(int64_t n)
{
    const int64_t g = (n + kOneBlock - 1) / kOneBlock;
    return (int)(g < 1 ? 1 : g > kMaxChunks ? kMaxChunks : g);
}

__global__ void __launch_bounds__(512)
count_kernel(const int32_t* __restrict__ ids, int32_t n, int32_t E, int64_t chunk, int32_t* __restrict__ hist)
{
    extern __shared__ int32_t cnt[];       // [E]
    for (int e = threadIdx.x; e < E; e += blockDim.x) cnt[e] = 0;
    __syncthreads();
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int64_t lo = blockIdx.x * chunk, hi = min((int64_t)n, lo + chunk);
#pragma unroll 8
    for (int64_t i = lo + threadIdx.x; i < hi; i += blockDim.x) {
        const int e = __ldg(ids + i);
        if (e >= 0 && e < E) atomicAdd(&cnt[e], 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < E; e += blockDim.x) hist[(int64_t)blockIdx.x * E + e] = cnt[e];
}

// Inclusive sum over the lanes of a warp.
__device__ __forceinline__ int scan32(int v, int lane)
{
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xFFFFFFFFu, v, o);
        if (lane >= o) v += u;
    }
    return v;
}

// Shared memory of place_kernel, in ints.  A row of `base` is an expert's counts per warp, one int longer than
// the warps: lanes over warps as well as lanes over experts touch different banks.
struct PlaceLayout {
    int base, total, before, first, local, delta, sums, order, all;
    __host__ __device__ explicit PlaceLayout(int E)
    {
        base = 0;
        total = E * (NW + 1);
        before = total + E;
        first = before + E;            // [E + 1]
        local = first + E + 1;         // [E] block's pairs before an expert's
        delta = local + E;             // [E] row of a block's pair minus its place in the block's order
        sums = delta + E;              // [2][32]
        order = sums + 64;             // [kOneBlock] the block's pairs in expert order
        all = order + (int)kOneBlock;
    }
};

// Launched while count_kernel runs (programmatic serialization): what needs only the ids comes first.
__global__ void __launch_bounds__(NW * 32)
place_kernel(const int32_t* __restrict__ ids, int32_t n, int32_t E, int32_t align, int64_t chunk,
             const int32_t* hist, int32_t* __restrict__ starts, int32_t* __restrict__ source,
             int32_t rows, int32_t* __restrict__ slot)
{
    extern __shared__ int32_t sm[];
    const PlaceLayout L(E);
    int32_t *base = sm + L.base, *total = sm + L.total, *before = sm + L.before, *first = sm + L.first;
    int32_t *local = sm + L.local, *delta = sm + L.delta, *sums = sm + L.sums, *order = sm + L.order;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    // without counts of chunks every block sorts all pairs, and all but the first only for the rows that no pair takes
    const int64_t lo = hist ? blockIdx.x * chunk : 0, hi = min((int64_t)n, lo + chunk);
    const int64_t piece = ((chunk + NW - 1) / NW + 31) / 32 * 32;
    const int64_t wlo = min(hi, lo + warp * piece), whi = min(hi, wlo + piece);
    const bool kept = piece <= KEEP * 32;  // a lane's ids stay in registers, the block's order in shared memory

    if (!hist) asm volatile("griddepcontrol.wait;" ::: "memory");
    for (int i = threadIdx.x; i < L.first; i += NW * 32) sm[i] = 0;
    int32_t mine[KEEP];
    if (kept) {
#pragma unroll
        for (int k = 0; k < KEEP; ++k) {
            const int64_t i = wlo + k * 32 + lane;
            mine[k] = i < whi ? __ldg(ids + i) : -1;
        }
    }
    __syncthreads();
    if (kept) {
#pragma unroll
        for (int k = 0; k < KEEP; ++k)
            if (mine[k] >= 0 && mine[k] < E) atomicAdd(&base[mine[k] * (NW + 1) + warp], 1);
    } else {
#pragma unroll 8
        for (int64_t i = wlo + lane; i < whi; i += 32) {
            const int e = __ldg(ids + i);
            if (e >= 0 && e < E) atomicAdd(&base[e * (NW + 1) + warp], 1);
        }
    }
    __syncthreads();
    // the block's pairs of an expert before each warp's, and all of them
    for (int e = warp; e < E; e += NW) {
        const int c = base[e * (NW + 1) + lane], s = scan32(c, lane);
        base[e * (NW + 1) + lane] = s - c;
        if (lane == 31) {
            local[e] = s;
            if (!hist) total[e] = s;
        }
    }
    if (hist) {
        asm volatile("griddepcontrol.wait;" ::: "memory");
        // thread (four experts, part) sums a part of the chunks: as many parts as the block has threads for
        const int G = (int)gridDim.x, quads = E / 4, parts = quads ? max(1, NW * 32 / quads) : 1;
        const bool vec = E % 4 == 0 && (uintptr_t)hist % 16 == 0;
        for (int u = threadIdx.x; vec && u < parts * quads; u += NW * 32) {
            const int part = u / quads, q = u - part * quads;
            int4 b = make_int4(0, 0, 0, 0), t = b;
#pragma unroll 4
            for (int c = part; c < G; c += parts) {
                const int4 h = *reinterpret_cast<const int4*>(hist + (int64_t)c * E + 4 * q);
                const bool early = c < (int)blockIdx.x;
                t.x += h.x; t.y += h.y; t.z += h.z; t.w += h.w;
                b.x += early ? h.x : 0; b.y += early ? h.y : 0; b.z += early ? h.z : 0; b.w += early ? h.w : 0;
            }
            atomicAdd(&total[4 * q], t.x); atomicAdd(&total[4 * q + 1], t.y); atomicAdd(&total[4 * q + 2], t.z); atomicAdd(&total[4 * q + 3], t.w);
            atomicAdd(&before[4 * q], b.x); atomicAdd(&before[4 * q + 1], b.y); atomicAdd(&before[4 * q + 2], b.z); atomicAdd(&before[4 * q + 3], b.w);
        }
        for (int k = threadIdx.x; !vec && k < E; k += NW * 32) {
            int b = 0, t = 0;
#pragma unroll 8
            for (int c = 0; c < G; ++c) {
                const int h = hist[(int64_t)c * E + k];
                t += h;
                b += c < (int)blockIdx.x ? h : 0;
            }
            total[k] = t;
            before[k] = b;
        }
    }
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    __syncthreads();
    // over the experts: warp w scans experts 32 w .., then adds the sums of the warps before it
    const int e = warp * 32 + lane;
    const int seg = e < E ? (total[e] + align - 1) / align * align : 0, cnt = e < E ? local[e] : 0;
    int seg_to = scan32(seg, lane), cnt_to = scan32(cnt, lane);
    if (lane == 31) {
        sums[warp] = seg_to;
        sums[32 + warp] = cnt_to;
    }
    __syncthreads();
    const int s0 = sums[lane], s1 = sums[32 + lane];
    const int t0 = scan32(s0, lane), t1 = scan32(s1, lane);
    seg_to += __shfl_sync(0xFFFFFFFFu, t0 - s0, warp);
    cnt_to += __shfl_sync(0xFFFFFFFFu, t1 - s1, warp);
    const int in_block = __shfl_sync(0xFFFFFFFFu, t1, 31);
    if (e < E) {
        first[e] = seg_to - seg;
        local[e] = cnt_to - cnt;
        delta[e] = seg_to - seg + before[e] - (cnt_to - cnt);
        if (e == E - 1) first[E] = seg_to;
    }
    __syncthreads();
    if (blockIdx.x == 0)
        for (int k = threadIdx.x; k <= E; k += NW * 32) starts[k] = first[k];
    // rows that no pair takes: behind each expert's pairs, and behind the last segment
    // (a block per expert where there are as many, else a warp)
    const bool by_block = (int)gridDim.x >= E;
    const int step = by_block ? NW * 32 : 32, from = by_block ? (int)threadIdx.x : lane;
    for (int k = (int)blockIdx.x + (by_block ? 0 : warp * (int)gridDim.x); k < E; k += (by_block ? 1 : NW) * (int)gridDim.x)
        for (int r = first[k] + total[k] + from; r < first[k + 1]; r += step) if (r < rows) source[r] = -1;
    for (int64_t r = (int64_t)first[E] + blockIdx.x * (NW * 32) + threadIdx.x; r < rows; r += (int64_t)gridDim.x * (NW * 32))
        source[r] = -1;
    if (!hist && blockIdx.x > 0) return;

    const int bits = 32 - __clz(E - 1);        // of an expert number (0 for E = 1)
    auto place = [&](int64_t i, int x) {
        if (x >= E || x < 0) x = -1;
        // lanes with my expert: one ballot per bit of its number (a match over 32 different numbers costs 32 rounds)
        unsigned same = __ballot_sync(0xFFFFFFFFu, x >= 0);
#pragma unroll
        for (int b = 0; b < 10; ++b) {
            if (b >= bits) break;
            const bool one = x & (1 << b);
            const unsigned set = __ballot_sync(0xFFFFFFFFu, one);
            same &= one ? set : ~set;
        }
        int r = -1;
        if (x >= 0) {
            const int k = local[x] + base[x * (NW + 1) + warp] + __popc(same & ((1u << lane) - 1u));
            r = k + delta[x];
            // the rows of the block's order are runs: written one by one, a warp's 32 would be 32 sectors
            if (kept) order[k] = x << 16 | (int)(i - lo);
            else if (r < rows) source[r] = (int32_t)i;
        }
        if (i < whi) slot[i] = r;
        __syncwarp();
        if (x >= 0 && (int)(__ffs(same) - 1) == lane) base[x * (NW + 1) + warp] += __popc(same);
        __syncwarp();
    };
    if (kept) {
#pragma unroll
        for (int k = 0; k < KEEP; ++k)
            if (wlo + k * 32 < whi) place(wlo + k * 32 + lane, mine[k]);
        __syncthreads();
        for (int k = threadIdx.x; k < in_block; k += NW * 32) {
            const int v = order[k], r = k + delta[v >> 16];
            if (r < rows) source[r] = (int32_t)lo + (v & 0xFFFF);
        }
    } else {
        for (int64_t i0 = wlo; i0 < whi; i0 += 32) place(i0 + lane, i0 + lane < whi ? __ldg(ids + i0 + lane) : -1);
    }
}

// ------------------------------------------------------------------------------------- rows
// A block's 256 threads are TY rows (or tokens) of TX threads, TX a power of two of 8..256.
using f8::Eight;
constexpr int kUnaligned = 2;              // rows in flight that need not begin on multiples of 16 bytes

template <int TYPE, bool VEC>
__global__ void __launch_bounds__(256)
gather_kernel(const ExpertRowsParams p, int tx_bits)
{
    f8::wait_for_predecessor();
    using T = typename f8::Elem<TYPE>::T;
    const int TX = 1 << tx_bits, tx = threadIdx.x & (TX - 1);
    const int64_t r = (int64_t)blockIdx.x * (256 >> tx_bits) + (threadIdx.x >> tx_bits);
    const bool mine = r < p.rows;
    if (VEC && !mine) return;
    const int pair = mine ? p.source[r] : -1, t = pair / p.topk;
    const bool on = pair >= 0 && t < p.tokens;
    const float w = on && p.w ? p.w[pair] : 1.0f;
    const T* src = static_cast<const T*>(p.X) + (on ? t * p.ldx : 0);
    T* dst = static_cast<T*>(p.out) + (mine ? r * p.ldo : 0);
    for (int c0 = 0; c0 < p.D; c0 += TX * 8) {             // whole warps
        const int c = c0 + tx * 8, left = mine ? p.D - c : 0, n = VEC ? left : max(0, min(8, left));
        f8::Coming<VEC, T> x;
        x.load(src + c, on ? n : 0, f8::careful_at(t, p.tokens, c, left, p.D));
        Eight<T> v = x.get(src + c, on ? n : 0);
        if (p.w) {
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = v.get(i) * w;
            f8::pack8(v, f);
        }
        f8::store8<VEC>(dst + c, left, v, tx, TX);
    }
}

// Row and weight of pair j0 + lane % J of a token, -1 where there is none: every J threads of a token hold its next J
// pairs between them.
struct Pair { int s; float w; };
template <int J> __device__ __forceinline__ Pair pair_of(const ExpertRowsParams& p, int64_t t, bool mine, int j0, int lane)
{
    const int j = j0 + lane % J;
    Pair q{-1, 1.0f};
    if (mine && j < p.topk) {
        q.s = __ldg(p.slot + t * p.topk + j);
        if (p.w) q.w = __ldg(p.w + t * p.topk + j);
    }
    return q;
}
template <int J> __device__ __forceinline__ void spread(const ExpertRowsParams& p, const Pair& q, int lane, int (&s)[J], float (&w)[J])
{
#pragma unroll
    for (int j = 0; j < J; ++j) {
        s[j] = __shfl_sync(0xFFFFFFFFu, q.s, lane / J * J + j);
        w[j] = __shfl_sync(0xFFFFFFFFu, q.w, lane / J * J + j);
        if (s[j] >= p.rows) s[j] = -1;
    }
}

// 16-bit types: four blocks per SM have 128 KB of rows in flight.
template <int TYPE, bool VEC>
__global__ void __launch_bounds__(256, VEC && TYPE == Q4_F32 ? 1 : 4)
combine_kernel(const ExpertRowsParams p, int tx_bits)
{
    f8::wait_for_predecessor();
    using T = typename f8::Elem<TYPE>::T;
    const int TX = 1 << tx_bits, tx = threadIdx.x & (TX - 1);
    const int64_t t = (int64_t)blockIdx.x * (256 >> tx_bits) + (threadIdx.x >> tx_bits);
    const int c = (blockIdx.y * TX + tx) * 8, lane = threadIdx.x & 31;
    const bool mine = t < p.tokens;
    const int left = mine ? p.D - c : 0, n = VEC ? left : max(0, min(8, left));
    // Rows in flight.  Unaligned ones take two pieces each and code that has to be fetched once per block: two at a time with four
    // blocks per SM 43 us for 4096 x 8 x 2047 (four and three 46, eight and two 56; aligned rows 24).
    constexpr int J = VEC ? 8 : kUnaligned;
    float acc[8] = {};
    Pair ahead = pair_of<J>(p, t, mine, 0, lane);
#pragma unroll 1
    for (int j0 = 0; j0 < p.topk; j0 += J) {
        int s[J];
        float w[J];
        f8::Coming<VEC, T> v[J];
        spread(p, ahead, lane, s, w);
        if (j0 + J < p.topk) ahead = pair_of<J>(p, t, mine, j0 + J, lane);
#pragma unroll
        for (int j = 0; j < J; ++j)
            v[j].load(static_cast<const T*>(p.Y) + (s[j] >= 0 ? s[j] * p.ldy + c : 0), s[j] >= 0 ? n : 0,
                      f8::careful_at(s[j], p.rows, c, left, p.D));
#pragma unroll
        for (int j = 0; j < J; ++j) {
            if (s[j] < 0) continue;                 // a dropped pair's weight may be anything
            const Eight<T> y = v[j].get(static_cast<const T*>(p.Y) + s[j] * p.ldy + c, n);
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[i] = fmaf(w[j], y.get(i), acc[i]);
        }
    }
    Eight<T> o;
    f8::pack8(o, acc);
    f8::store8<VEC>(static_cast<T*>(p.out) + (VEC || mine ? t * p.ldo + c : 0), left, o, tx, TX);
}

// Sums of eight values over the 32 lanes of a warp; lane l < 8 returns the sum of value l.  Each step
// halves the values and doubles the lanes that were summed: 9 shuffles instead of 40.
__device__ __forceinline__ float reduce8(float (&d)[8], int lane)
{
#pragma unroll
    for (int b = 4; b; b >>= 1) {
        const bool up = lane & b;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (j >= b) break;
            const float give = up ? d[j] : d[j + b];
            d[j] = (up ? d[j + b] : d[j]) + __shfl_xor_sync(0xFFFFFFFFu, give, b);
        }
    }
    d[0] += __shfl_xor_sync(0xFFFFFFFFu, d[0], 8);
    return d[0] + __shfl_xor_sync(0xFFFFFFFFu, d[0], 16);
}

// By tokens: a token's gradient is read once, its rows wherever they lie.  (By rows of the experts' side, read and
// written front to back with the gradients from L2, 4096 x 8 x 2048 takes 68 us instead of 60: the streams push the
// gradients out of L2.  Rows that happen to lie in token order take 48: the rest is the scattered writes.)
// SPREAD (unaligned rows): a token's pairs are shared by as many blocks as have two of them each.
template <int TYPE, bool VEC, bool SPREAD>
__global__ void __launch_bounds__(256, VEC && TYPE == Q4_F32 ? 2 : 3)
combine_grad_kernel(const ExpertRowsParams p, int tx_bits, int token_blocks)
{
    f8::wait_for_predecessor();
    using T = typename f8::Elem<TYPE>::T;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if ((int)blockIdx.x >= token_blocks) {
        // rows that belong to no pair get zeros: 32 rows per warp
        constexpr int PV = 16 / (int)sizeof(T);
        const int64_t r0 = ((int64_t)blockIdx.x - token_blocks) * 256 + warp * 32;
        const int pair = r0 + lane < p.rows ? p.source[r0 + lane] : 0;
        const bool absent = r0 + lane < p.rows && (pair < 0 || pair / p.topk >= p.tokens);
        for (unsigned none = __ballot_sync(0xFFFFFFFFu, absent); none; none &= none - 1) {
            T* const dst = static_cast<T*>(p.out) + (r0 + __ffs(none) - 1) * p.ldo;
            const int head = min((int)(-(uintptr_t)dst & 15) / (int)sizeof(T), p.D), body = (p.D - head) / PV;
            for (int k = lane; k < body; k += 32) __stcs(reinterpret_cast<uint4*>(dst + head) + k, make_uint4(0, 0, 0, 0));
            const int rest = p.D - body * PV;              // values before and behind the pieces of 16 bytes
            if (lane < rest) dst[lane < head ? lane : lane + body * PV] = f8::from_f<T>(0.0f);
        }
        return;
    }
    // Rows in flight.  Unaligned: two with three blocks per SM 121 us for 4096 x 8 x 2047 (four and two 143, one and four 184;
    // aligned rows 59): issue binds, a row's cut and put-together pieces are three times an aligned one's instructions.
    constexpr int J = VEC ? 8 : kUnaligned;
    __shared__ float part[8][8];
    const int TX = 1 << tx_bits, tx = threadIdx.x & (TX - 1), TY = 256 >> tx_bits, ty = threadIdx.x >> tx_bits;
    // a block walks groups of TY tokens (SPREAD: J pairs of each, other blocks the others); the next group's pairs are
    // loaded before this one's rows
    const int parts = SPREAD ? (p.topk + J - 1) / J : 1;
    const int from = SPREAD ? (int)blockIdx.x % parts * J : 0, to = SPREAD ? min(p.topk, from + J) : p.topk;
    int64_t t = (int64_t)(blockIdx.x / (unsigned)parts) * TY + ty;
    const int64_t step = (int64_t)(token_blocks / parts) * TY;
    Pair ahead = pair_of<J>(p, t, t < p.tokens, from, lane);
    for (int64_t group = t - ty; group < p.tokens; group += step, t += step) {
        const bool mine = t < p.tokens;
        const T* g = static_cast<const T*>(p.X) + (mine ? t * p.ldx : 0);
#pragma unroll 1
        for (int j0 = from; j0 < to; j0 += J) {
            int s[J];
            float w[J], dot[8] = {};
            spread(p, ahead, lane, s, w);
            const bool more = !SPREAD && j0 + J < to;
            const int64_t t_next = more ? t : t + step;
            ahead = pair_of<J>(p, t_next, t_next < p.tokens, more ? j0 + J : from, lane);
            auto columns = [&](auto careful) {
                constexpr bool CAREFUL = decltype(careful)::value;
                // (rows of any alignment: whole warps go on together)
                for (int c = tx * 8; VEC ? mine && c < p.D : c - tx * 8 < p.D; c += TX * 8) {
                    const int left = VEC || mine ? p.D - c : 0, n = VEC ? left : max(0, min(8, left));
                    f8::Coming<VEC, T> dc;
                    dc.load(g + c, n, CAREFUL && f8::careful_at(t, p.tokens, c, left, p.D));
                    f8::Coming<VEC, T> yc[J];
#pragma unroll
                    for (int j = 0; j < J; ++j)
                        yc[j].load(static_cast<const T*>(p.Y) + (s[j] >= 0 ? s[j] * p.ldy + c : 0), s[j] >= 0 ? n : 0,
                                   CAREFUL && f8::careful_at(s[j], p.rows, c, left, p.D));
                    const Eight<T> d = dc.template get<CAREFUL>(g + c, n);
#pragma unroll
                    for (int j = 0; j < J; ++j) {
                        if (VEC ? s[j] < 0 : __all_sync(0xFFFFFFFFu, s[j] < 0)) continue;
                        const Eight<T> y = yc[j].template get<CAREFUL>(static_cast<const T*>(p.Y) + (s[j] >= 0 ? s[j] * p.ldy + c : 0), VEC || s[j] >= 0 ? n : 0);
                        float o[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            dot[j] = fmaf(d.get(i), y.get(i), dot[j]);
                            o[i] = w[j] * d.get(i);
                        }
                        Eight<T> e;
                        f8::pack8(e, o);
                        f8::store8<VEC>(static_cast<T*>(p.out) + (VEC || s[j] >= 0 ? s[j] * p.ldo + c : 0), VEC || s[j] >= 0 ? left : 0, e, tx, TX);
                    }
                }
            };
            // Many unaligned tokens: rows without careful values go through code without the call that reads them, whose
            // place among the rows in flight costs registers (132 us with it, 121 without)
            bool edge = VEC || SPREAD || t == 0 || t == p.tokens - 1 || p.D < 16;
#pragma unroll
            for (int j = 0; j < J; ++j) edge = edge || s[j] == 0 || s[j] == p.rows - 1;
            if (VEC || SPREAD || __any_sync(0xFFFFFFFFu, edge)) columns(std::true_type{});
            else columns(std::false_type{});
            // an absent pair beside a present one of the warp's other tokens: what its dOut times nothing came to
            // (NaN, if dOut is not finite) does not count
#pragma unroll
            for (int j = 0; j < J; ++j)
                if (!VEC && s[j] < 0) dot[j] = 0.0f;
            if (TX >= 32) {
                const float sum = reduce8(dot, lane);
                if (lane < 8) part[warp][lane] = sum;
                __syncthreads();
                if (tx < J) {
                    float all = 0.0f;
                    for (int k = 0; k < TX / 32; ++k) all += part[warp + k][tx];
                    if (mine && j0 + tx < p.topk) p.dw[t * p.topk + j0 + tx] = all;
                }
                __syncthreads();
            } else {
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    for (int o = TX >> 1; o; o >>= 1) dot[j] += __shfl_xor_sync(0xFFFFFFFFu, dot[j], o);
                    if (tx == 0 && mine && j0 + j < p.topk) p.dw[t * p.topk + j0 + j] = dot[j];
                }
            }
        }
    }
}

static int tx_bits_of(int D)
{
    int b = 3;
    while (b < 8 && (8 << b) < D) ++b;
    return b;
}

}  // namespace experts

using namespace experts;

// The instance of a row kernel for the call's type and alignment.
#define Q4_ROWS_LAUNCH(kernel, grid, ...)                                                                        \
    (p.type == Q4_F32    ? f8::launch(p.vec ? kernel<Q4_F32, true> : kernel<Q4_F32, false>, grid, 256, 0, st, __VA_ARGS__)    \
     : p.type == Q4_BF16 ? f8::launch(p.vec ? kernel<Q4_BF16, true> : kernel<Q4_BF16, false>, grid, 256, 0, st, __VA_ARGS__)  \
                         : f8::launch(p.vec ? kernel<Q4_F16, true> : kernel<Q4_F16, false>, grid, 256, 0, st, __VA_ARGS__))

size_t expert_sort_ws_bytes(int64_t n, int32_t E)
{
    const int g = chunks_of(n);
    return g == 1 ? 0 : (size_t)g * (size_t)E * 4;
}

cudaError_t launch_expert_sort(const int32_t* ids, int32_t n, int32_t E, int32_t align, int32_t* starts, int32_t* source,
                               int32_t rows, int32_t* slot, void* ws, cudaStream_t st)
{
    const int g = chunks_of(n);
    const int64_t chunk = ((int64_t)n + g - 1) / g;
    const size_t smem = (size_t)PlaceLayout(E).all * 4;
    if (smem > 48 * 1024) {
        // the limit belongs to the device, not to the call: set once, to the most experts' size, so that a call of fewer
        // on another host thread does not lower it between this one's setting and its launch
        static bool ready[64] = {};
        int dev = 0;
        const cudaError_t at = cudaGetDevice(&dev);
        if (at != cudaSuccess) return at;
        if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
        if (!ready[dev]) {
            const cudaError_t e = cudaFuncSetAttribute(place_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, PlaceLayout(Q4_MAX_EXPERTS).all * 4);
            if (e != cudaSuccess) return e;
            ready[dev] = true;
        }
    }
    int32_t* hist = static_cast<int32_t*>(ws);
    if (g > 1) {
        const cudaError_t err = f8::launch(count_kernel, (unsigned)g, 512, (size_t)E * 4, st, ids, n, E, chunk, hist);
        if (err != cudaSuccess) return err;
    }
    // one block's pairs: rows that no pair takes are shared by more blocks (2984 pairs, 256 experts, align 128, 32512 such
    // rows: 10.0 us by one block, 7.4 by all; 512 rows per block are no faster than 2048)
    const int64_t free_rows = (int64_t)rows - n;
    const unsigned blocks = g > 1 ? (unsigned)g : 1u + (unsigned)(free_rows <= 0 ? 0 : free_rows / kRowsPerBlock < 63 ? free_rows / kRowsPerBlock : 63);
    return f8::launch(place_kernel, blocks, NW * 32, smem, st, ids, n, E, align, chunk,
                      (const int32_t*)(g > 1 ? hist : nullptr), starts, source, rows, slot);
}

cudaError_t launch_expert_gather(const ExpertRowsParams& p, cudaStream_t st)
{
    const int b = tx_bits_of(p.D), ty = 256 >> b;
    const unsigned grid = (unsigned)(((int64_t)p.rows + ty - 1) / ty);
    return Q4_ROWS_LAUNCH(gather_kernel, grid, p, b);
}

cudaError_t launch_expert_combine(const ExpertRowsParams& p, cudaStream_t st)
{
    const int b = tx_bits_of(p.D), ty = 256 >> b;
    const dim3 grid((unsigned)(((int64_t)p.tokens + ty - 1) / ty), (unsigned)((p.D + (8 << b) - 1) / (8 << b)));
    return Q4_ROWS_LAUNCH(combine_kernel, grid, p, b);
}

cudaError_t launch_expert_combine_grad(const ExpertRowsParams& p, cudaStream_t st)
{
    const int b = tx_bits_of(p.D), ty = 256 >> b;
    const int64_t groups = ((int64_t)p.tokens + ty - 1) / ty;
    // Blocks that walk the tokens: three per SM, as many as are resident; of aligned float32 rows (128 registers) two are, and
    // four take two rounds whose second evens out the first's ends (two, three and four: 4096 x 8 x 2048 94, 111 and 94 us,
    // 1000 x 8 x 2048 28.4, 29.2 and 27.7; bfloat16 4096 x 8 x 2048 56, 48 and 56).
    const int blocks = 2 * f8_pairs_of_device() * (p.vec && p.type == Q4_F32 ? 4 : 3);
    // Unaligned rows: a token's pairs over several blocks while the tokens alone do not keep the blocks evenly busy.  From five
    // rounds on the gradients that such blocks read again, and the calls for their edges, cost more: with and without,
    // 6 x 8 x 101 3.4 and 9.5 us, 600 x 8 x 2047 21.6 and 27.7, 2048 x 8 x 2047 64 and 67, 2220 x 8 x 2047 70 and 68, 4096 x 8 x 2047
    // 127 and 121, 8192 x 8 x 2047 251 and 238; float32 4096 x 8 x 2047 155 and 145.
    const bool spread = !p.vec && groups < 5 * blocks;
    const int parts = spread ? (p.topk + kUnaligned - 1) / kUnaligned : 1, most = blocks > parts ? blocks / parts : 1;
    const int tb = (int)(groups < most ? groups : most) * parts;
    const unsigned grid = (unsigned)(tb + ((int64_t)p.rows + 255) / 256);
    const auto run = [&](auto aligned, auto shared, auto whole) { return f8::launch(p.vec ? aligned : spread ? shared : whole, grid, 256, 0, st, p, b, tb); };
    if (p.type == Q4_F32) return run(combine_grad_kernel<Q4_F32, true, false>, combine_grad_kernel<Q4_F32, false, true>, combine_grad_kernel<Q4_F32, false, false>);
    if (p.type == Q4_BF16) return run(combine_grad_kernel<Q4_BF16, true, false>, combine_grad_kernel<Q4_BF16, false, true>, combine_grad_kernel<Q4_BF16, false, false>);
    return run(combine_grad_kernel<Q4_F16, true, false>, combine_grad_kernel<Q4_F16, false, true>, combine_grad_kernel<Q4_F16, false, false>);
}

}  // namespace q4
