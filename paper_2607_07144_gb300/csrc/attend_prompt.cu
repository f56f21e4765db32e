// Attention over the paged 8- and 4-bit cache for many rows a KV head (attend.cu has
// the mathematics): both products on the 5th-generation tensor cores.
//
// A block takes 256 rows of one KV head (its query heads, times new tokens) and
// walks its share of the keys in tiles of 128.  Four warps load the pages' codes
// and write them as fp16 tiles to shared memory (codes are exact in fp16; each
// tile is converted once for 256 rows), one thread issues the tcgen05.mma, and
// two groups of four warps, a thread a row, do the softmax of 128 rows each: the
// one's products run while the other exponentiates.  S = Q K^T and then P (fp16,
// in place of S) and O stay in tensor memory: P is the second product's first
// operand from there, and V is read as it lies, [key][dimension], by a transposed
// descriptor.  A tile is read once, against the row's reference exponent from the
// tiles before: only when weights come out above 2^15 does the reference move up
// to the largest score seen (O and what has been written of P are then scaled by
// the power of two between them, exactly but for weights that become subnormal in
// fp16, 2^-20 of the largest and less), so no pass looks for the maximum.
//
// Two pieces of 4,096 tokens against 12-16k positions, 8 heads of 128 with 4 query
// heads each: 1,383 us, 1.38 PFLOP/s, bound by a group's round of scores, softmax
// and product (3.5k cycles a tile, of which the products of both groups are 2.1k).
// 13 prompts of 1 to 1,000 tokens, 12 heads of 64: 39 us, bound by the start and
// the end of a block.
//
// 4-bit pages: a key, middle + (c - 7.5) step, is (c - 8) step, whose 11 bits fp16 holds,
// and middle + step / 2 in every dimension.  K's tile holds the former over the power of
// two that brings the largest of 16 keys' 8 step + |middle| to [2^14, 2^15), the unit's
// scale (steps and middles below 2^-30 of that are rounded to multiples of fp16's 2^-24, 2^-38
// of it); the latter times the query's sum is a step of 16 more dimensions: middle, middle,
// step / 2, step / 2 against the sum's upper and lower half, twice, which leave out 2^-22 of
// the sum: an error of 2^-22 |middle sum q|, next to fp32's of as large a product.  So scores
// come out as over 8-bit pages, without a number of the key's in the softmax (with two there,
// 8 bytes of shared memory a score: 2,334 us against 1,678).  V's tile holds whole values over such a power of two, rounded to fp16
// once, as the weights are (for bfloat16 outputs; see EXACT).  Eight codes of a word lie in a
// tile in the order 0 4 1 5 2 6 3 7, as masks give them two at a time; so do the queries'
// elements, and the outputs' are put back.
//
// The pieces above: 1,692 us, 1.13 PFLOP/s (float16 1,872), GPT-2-shaped prompts 47 us (float16);
// 15 us of it are what keeps numbers of masked positions out (1,678 before).  Without the codes'
// loads 1,471: a shuffle behind a load in flight waits for it, so that an iteration's come before
// its loads (1,682 against 2,138); with the table's look-up left for the
// iteration after 2,134.  Seven warps convert instead of four, all with the same statements:
// those for K and V apart compete for the instruction cache.
#include "attend.cuh"

using namespace fkvd;

namespace {

constexpr int kRows = 256, kThreads = 512;
constexpr float kPBits = 6.0f;          // a reference gives its own score the weight 2^6
constexpr float kMostSum = 32768.0f;    // of 64 weights: each then fits fp16

template <int D> struct PromptShape {
    static constexpr int half = 128 * 128;                   // 64 dimensions of 128 rows in fp16
    static constexpr int tile = half * (D / 64);             // 128 rows
    static constexpr int off_q = 0, off_k = 2 * tile, off_v = 4 * tile, off_n = 6 * tile;
    // 4-bit pages: 16 more dimensions of two tiles of keys, then of the groups' queries, 32 bytes each of 128-byte rows
    // (and of four tiles' values what all dimensions of a key have, see EXACT)
    static constexpr int off_h = off_n + half;
    static constexpr int smem(int format) { return (format == FKV_UINT4 ? off_h + 4 * 128 * 4 : off_n) + 1024; }
};

enum { K_FULL = 0, K_EMPTY = 2, V_FULL = 4, V_EMPTY = 6, SC_FULL = 8, S_FULL = 12, P_FULL = 14, O_FULL = 16, Q_FULL = 18,
       DRAIN = 19, N_BARS = 20 };

__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float *r)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]), "=f"(r[9]), "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15]), "=f"(r[16]), "=f"(r[17]), "=f"(r[18]), "=f"(r[19]), "=f"(r[20]), "=f"(r[21]), "=f"(r[22]), "=f"(r[23]), "=f"(r[24]), "=f"(r[25]), "=f"(r[26]), "=f"(r[27]), "=f"(r[28]), "=f"(r[29]), "=f"(r[30]), "=f"(r[31])
                 : "r"(taddr)
                 : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t *r)
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
                 "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
                 : "memory");
}
// Waits for this thread's loads; the registers pass through, so that nothing
// reads them earlier.
__device__ __forceinline__ void tmem_wait_ld(float *r)
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+f"(r[0]), "+f"(r[1]), "+f"(r[2]), "+f"(r[3]), "+f"(r[4]), "+f"(r[5]), "+f"(r[6]), "+f"(r[7]), "+f"(r[8]), "+f"(r[9]), "+f"(r[10]), "+f"(r[11]), "+f"(r[12]), "+f"(r[13]), "+f"(r[14]), "+f"(r[15]), "+f"(r[16]), "+f"(r[17]), "+f"(r[18]), "+f"(r[19]), "+f"(r[20]), "+f"(r[21]), "+f"(r[22]), "+f"(r[23]), "+f"(r[24]), "+f"(r[25]), "+f"(r[26]), "+f"(r[27]), "+f"(r[28]), "+f"(r[29]), "+f"(r[30]), "+f"(r[31])
                 :
                 : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t *r)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n\t"
                 "tcgen05.wait::ld.sync.aligned;"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(taddr)
                 : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ void mbar_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}

__device__ __forceinline__ bool elect_one()
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}

// A tile's MMAs are one statement each, from the low words of the first step's
// descriptors (a descriptor's address counts 16 bytes, its high word is the
// layout): the issuing warp shares its scheduler with five working ones, and what
// it executes between two MMAs is what the tensor core waits for.  Measured beside
// twenty busy warps: 161 cycles an MMA issued by a lane picked by its number, 89
// by an elected one with 64-bit descriptors, 79 like this, of which the tensor
// core itself takes 64.
//
// D[tmem] = A[smem] B[smem]^T over D dimensions: 128-byte swizzled rows of 64.
template <int D> __device__ __forceinline__ void umma_tile_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc)
{
    if (D == 128)
        asm volatile(
            "{\n\t.reg .b64 x, y;\n\t.reg .b32 p, q, hi;\n\t.reg .pred f, t;\n\t"
            "mov.b32 hi, 0x40004040;\n\tsetp.ne.b32 f, 0, 0;\n\tsetp.eq.b32 t, 0, 0;\n\t"
            "mov.b64 x, {%1, hi};\n\tmov.b64 y, {%2, hi};\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, f;\n\t"
            "add.u32 p, %1, 2;\n\tadd.u32 q, %2, 2;\n\tmov.b64 x, {p, hi};\n\tmov.b64 y, {q, hi};\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, t;\n\t"
            "add.u32 p, %1, 4;\n\tadd.u32 q, %2, 4;\n\tmov.b64 x, {p, hi};\n\tmov.b64 y, {q, hi};\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, t;\n\t"
            "add.u32 p, %1, 6;\n\tadd.u32 q, %2, 6;\n\tmov.b64 x, {p, hi};\n\tmov.b64 y, {q, hi};\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, t;\n\t"
            "add.u32 p, %1, 1024;\n\tadd.u32 q, %2, 1024;\n\tmov.b64 x, {p, hi};\n\tmov.b64 y, {q, hi};\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, t;\n\t"
            "add.u32 p, %1, 1026;\n\tadd.u32 q, %2, 1026;\n\tmov.b64 x, {p, hi};\n\tmov.b64 y, {q, hi};\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, t;\n\t"
            "add.u32 p, %1, 1028;\n\tadd.u32 q, %2, 1028;\n\tmov.b64 x, {p, hi};\n\tmov.b64 y, {q, hi};\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, t;\n\t"
            "add.u32 p, %1, 1030;\n\tadd.u32 q, %2, 1030;\n\tmov.b64 x, {p, hi};\n\tmov.b64 y, {q, hi};\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, t;\n\t"
            "}" ::"r"(d), "r"(a), "r"(b), "r"(idesc) : "memory");
    else
        asm volatile(
            "{\n\t.reg .b64 x, y;\n\t.reg .b32 p, q, hi;\n\t.reg .pred f, t;\n\t"
            "mov.b32 hi, 0x40004040;\n\tsetp.ne.b32 f, 0, 0;\n\tsetp.eq.b32 t, 0, 0;\n\t"
            "mov.b64 x, {%1, hi};\n\tmov.b64 y, {%2, hi};\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, f;\n\t"
            "add.u32 p, %1, 2;\n\tadd.u32 q, %2, 2;\n\tmov.b64 x, {p, hi};\n\tmov.b64 y, {q, hi};\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, t;\n\t"
            "add.u32 p, %1, 4;\n\tadd.u32 q, %2, 4;\n\tmov.b64 x, {p, hi};\n\tmov.b64 y, {q, hi};\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, t;\n\t"
            "add.u32 p, %1, 6;\n\tadd.u32 q, %2, 6;\n\tmov.b64 x, {p, hi};\n\tmov.b64 y, {q, hi};\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, t;\n\t"
            "}" ::"r"(d), "r"(a), "r"(b), "r"(idesc) : "memory");
}

// D[tmem] (+)= A[tmem] B[smem] over 128 keys: A fp16 pairs in 32-bit columns, B
// 16 keys (2048 bytes) a step.
__device__ __forceinline__ void umma_tile_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t accumulate,
                                             uint32_t b_hi)
{
    asm volatile(
        "{\n\t.reg .b64 y;\n\t.reg .b32 p, q;\n\t.reg .pred f, t;\n\t"
        "setp.ne.b32 f, %4, 0;\n\tsetp.eq.b32 t, 0, 0;\n\t"
        "mov.b32 p, %1;\n\tmov.b64 y, {%2, %5};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [p], y, %3, f;\n\t"
        "add.u32 p, %1, 8;\n\tadd.u32 q, %2, 128;\n\tmov.b64 y, {q, %5};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [p], y, %3, t;\n\t"
        "add.u32 p, %1, 16;\n\tadd.u32 q, %2, 256;\n\tmov.b64 y, {q, %5};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [p], y, %3, t;\n\t"
        "add.u32 p, %1, 24;\n\tadd.u32 q, %2, 384;\n\tmov.b64 y, {q, %5};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [p], y, %3, t;\n\t"
        "add.u32 p, %1, 32;\n\tadd.u32 q, %2, 512;\n\tmov.b64 y, {q, %5};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [p], y, %3, t;\n\t"
        "add.u32 p, %1, 40;\n\tadd.u32 q, %2, 640;\n\tmov.b64 y, {q, %5};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [p], y, %3, t;\n\t"
        "add.u32 p, %1, 48;\n\tadd.u32 q, %2, 768;\n\tmov.b64 y, {q, %5};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [p], y, %3, t;\n\t"
        "add.u32 p, %1, 56;\n\tadd.u32 q, %2, 896;\n\tmov.b64 y, {q, %5};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [p], y, %3, t;\n\t"
        "}" ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(accumulate), "r"(b_hi) : "memory");
}

// A [keys][dimensions] tile as the second operand with its dimensions outermost:
// 64 dimensions a 128-byte swizzled row, 8 keys a 1024-byte atom; the next 64
// dimensions `half` bytes on.
__device__ __forceinline__ uint64_t sdesc_mn_sw128(uint32_t saddr, uint32_t half)
{
    uint64_t d = 0;
    d |= static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4);
    d |= static_cast<uint64_t>(half >> 4) << 16;
    d |= static_cast<uint64_t>(1024 >> 4) << 32;
    d |= static_cast<uint64_t>(1) << 46;
    d |= static_cast<uint64_t>(2) << 61;
    return d;
}

__device__ __forceinline__ void sts128(uint32_t a, uint32_t x, uint32_t y, uint32_t z, uint32_t w)
{
    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(a), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}

// Eight 4-bit codes of a word as values, fp16 pairs (0, 4), (1, 5), (2, 6) and (3, 7), rounded
// once: (c - less) step + add.  A code at bits 4 to 7 of an fp16 number with an exponent of 6
// is 64 + c, exactly, and less 64 and 7.5 or 8 as well.
__device__ __forceinline__ void codes8_half(uint32_t w, __half2 less, __half2 step, __half2 add, uint32_t *f)
{
    const uint32_t x[4] = {w << 4, w, w >> 4, w >> 8};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t y = (x[i] & 0x00f000f0u) | 0x54005400u;
        const __half2 z = __hfma2(__hsub2(*reinterpret_cast<const __half2 *>(&y), less), step, add);
        f[i] = *reinterpret_cast<const uint32_t *>(&z);
    }
}
__device__ __forceinline__ uint32_t half2_bits(const __half2 &h) { return *reinterpret_cast<const uint32_t *>(&h); }

// The word whose first n bits are set (none for n <= 0, all for n >= 32).
__device__ __forceinline__ uint32_t below(int n)
{
    return static_cast<uint32_t>((1ull << max(0, min(32, n))) - 1);
}

// One group's softmax of a tile: see k_attend_prompt.
struct Row {
    float m, l;                 // reference exponent and the sum of weights
    float down;                 // what a score is multiplied by for the row's power of two
    int p, hi, from, pre;       // position and visible keys
    float slope;
    float mid;                  // EXACT: the weighted sum of what all dimensions of a value have
};

// What is done to a score: nothing; a cap that is plain (attend.cuh), a bias by
// distance, or both; a larger cap, and a bias if there is one.  (Together in one
// variant the larger caps' code costs the others 4 %.)
enum { SCORES_PLAIN, SCORES_GENERAL, SCORES_LARGE_CAP };

template <int D, int FMT, typename T, int SCORES>
__global__ void __launch_bounds__(kThreads, 1) k_attend_prompt(const AttendArgs a)
{
    using S = PromptShape<D>;
    constexpr bool GEN = SCORES != SCORES_PLAIN, FOUR = FMT == FKV_UINT4;
    // Outputs of 11 bits show a rounding of V as much as that of the weights: for them V's
    // tile, too, holds (c - 8) step, exactly, and the weighted sum of middle + step / 2 is
    // kept in fp32 beside the sum of weights.
    constexpr bool EXACT = FOUR && std::is_same<T, __half>::value;
    extern __shared__ uint8_t raw[];
    __shared__ __align__(8) uint64_t bars[N_BARS];
    // of the last four tiles' units of 16 keys: the scores' multiplier; log2 vs and share_of(vs)
    __shared__ float k_scales[4][8];
    __shared__ float2 v_scales[4][8];
    __shared__ uint32_t tmem_slot;
    __shared__ Seen rows_see;              // for the converters' look-ups: registers are short
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, group = warp >> 2;
    const uint32_t sbase = (smem_u32(raw) + 1023) & ~1023u;
    auto bar = [&](int i) { return smem_u32(bars) + 8 * i; };

    // the last rows of a causal prompt see the most keys: they go first
    int x = blockIdx.x;
    const int h = x % a.H;
    x /= a.H;
    const int split = x % a.splits;
    x /= a.splits;
    const int r = x % a.n_req, rt = a.row_tiles - 1 - x / a.n_req;
    Request q;
    if (!q.load(a, r)) {
        if (tid == 0)
            atomicOr(a.status, FKV_ST_RANGE);
        return;
    }
    const int rows = q.nq * a.G, row0 = rt * kRows;
    if (row0 >= rows)
        return;
    const int groups = rows - row0 > 128 ? 2 : 1;
    const int pa = q.p0 + static_cast<int>(a.gdiv.div(row0));
    const int pb = q.p0 + static_cast<int>(a.gdiv.div(min(row0 + kRows, rows) - 1));
    const Tiles tiles(a, q, pa, pb);
    const int i0 = split * a.chunk, n_it = max(0, min(tiles.n, i0 + a.chunk) - i0);
    // A bias by distance grows along the keys, and the reference with it, tile by
    // tile: general scores are walked from the last tile back (two pieces of 4,096
    // tokens against 12-16k positions, 8 heads of 128: 3,360 us forwards, 1,670 so; with
    // a cap of 30 2,580 and 2,610).
    auto tile_at = [&](int j) { return tiles.at(i0 + (GEN ? n_it - 1 - j : j)); };
    // the first group's rows end earlier: tiles at the share's end that none of
    // them sees are the second group's alone
    int n_first = n_it;
    if (groups == 2 && !GEN) {
        const Tiles own(a, q, pa, q.p0 + static_cast<int>(a.gdiv.div(row0 + 127)));
        while (n_first > 0 && tiles.at(i0 + n_first - 1) * kTile >= own.lim)
            --n_first;
    }

    if (tid == 0) {
        rows_see = tiles.seen;
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(K_FULL + i), FOUR ? 3 : 2);
            mbar_init(bar(K_EMPTY + i), 1);
            mbar_init(bar(V_FULL + i), FOUR ? 4 : 2);
            mbar_init(bar(V_EMPTY + i), 1);
            mbar_init(bar(S_FULL + i), 1);
            mbar_init(bar(P_FULL + i), 4);
            mbar_init(bar(O_FULL + i), 1);
        }
        for (int i = 0; i < 4; ++i)
            mbar_init(bar(SC_FULL + i), FOUR ? 7 : 4);
        mbar_init(bar(Q_FULL), 128 * groups);
        mbar_init(bar(DRAIN), 1);
        fence_mbar_init();
    }
    if (warp == 12)
        tmem_alloc(smem_u32(&tmem_slot), 512);
    if (FOUR) {
        // (most of the 16 dimensions are no one's)
        for (int i = tid; i < S::half / 16; i += kThreads)
            sts128(sbase + S::off_n + 16 * i, 0, 0, 0, 0);
        fence_proxy_async_smem();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;

    float *const v_mids = reinterpret_cast<float *>(raw + (sbase - smem_u32(raw)) + S::off_h);
    // 4-bit codes to fp16 tiles: a warp's n (2 or 3) units of 16 keys from u0 on, of K or V.
    // What 16 keys share, and every row's numbers, are one lane's a key; ids, codes and numbers
    // are asked for as 8-bit pages' are below.
    auto convert4 = [&](bool v_side, int u0, int n) {
        constexpr int C = D / 32, RP = 32 / C, NL = 16 / RP;       // 16-byte pieces of a row, rows at a time, loads a unit
        // eight lanes that store together hold the same piece of eight rows: other banks each
        const int c = lane / RP, r0 = lane % RP;
        const uint8_t *const pool = static_cast<const uint8_t *>(v_side ? a.pool_v : a.pool_k) + h * a.sh + c * 16 + r0 * a.st;
        const uint32_t *const numbers = reinterpret_cast<const uint32_t *>(v_side ? a.vs : a.ks) + h * a.sch;
        const float mul0 = score_multiplier(a, fabsf(a.scale));
        const int full_bar = v_side ? V_FULL : K_FULL, empty_bar = v_side ? V_EMPTY : K_EMPTY;
        const uint32_t at0 = sbase + (v_side ? S::off_v : S::off_k) + (c >> 1) * S::half + (16 * u0 + r0) * 128;
        const uint32_t sw = static_cast<uint32_t>((4 * (c & 1)) ^ (r0 & 7)) * 16;
        const bool whole = v_side && !EXACT;   // values, middle and all
        const __half2 less = __half2half2(__ushort_as_half(whole ? 0x5478 : 0x5480));         // 71.5, 72
        bool bad = false, ok = true;           // (ok: see the softmax's)
        auto first = [&](int j) { return tile_at(j) * kTile + 16 * u0; };
        struct Page {
            int id;
            bool on;
        };
        auto ask = [&](int j) {
            const int key = first(j) + 16 * lane;
            Page p = {-1, j < n_it && lane < n && rows_see.of(key)};
            if (p.on)
                p.id = a.table[r * a.table_stride + a.div.div(key)];
            return p;
        };
        auto check = [&](const Page &p) {
            if (p.on && (p.id < 0 || p.id >= a.n_blocks)) {
                bad = true;
                return 0;
            }
            return p.id;
        };
        uint4 v[3][NL];
        uint32_t num[2];                       // of keys lane and 32 + lane % 16; 0: not looked at
        auto load = [&](uint4 (&x)[3][NL], int j, int id) {
            int64_t from = -1, from_n = -1;
            if (id >= 0) {
                const int key = first(j) + 16 * lane, off = key - static_cast<int>(a.div.div(key)) * a.block;
                from = id * a.sb + off * a.st, from_n = id * a.scb + off;
            }
            // all of them before the first load: a shuffle behind one waits for it as well
            int64_t at[3], at_n[2];
#pragma unroll
            for (int u = 0; u < 3; ++u)
                at[u] = __shfl_sync(~0u, from, u);
            at_n[0] = __shfl_sync(~0u, from_n, lane >> 4), at_n[1] = __shfl_sync(~0u, from_n, 2);
#pragma unroll
            for (int u = 0; u < 3; ++u)
#pragma unroll
                for (int i = 0; i < NL; ++i)
                    x[u][i] = at[u] >= 0 ? __ldg(reinterpret_cast<const uint4 *>(pool + at[u] + i * RP * a.st)) : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int y = 0; y < 2; ++y)
                num[y] = at_n[y] >= 0 && first(j) + (y ? 32 + (lane & 15) : lane) < tiles.lim ? __ldg(numbers + at_n[y] + (lane & 15)) : 0;
        };
        const Page start = ask(0);
        Page after = ask(1);
        load(v, 0, check(start));
        int nid = check(after);
        for (int j = 0; j < n_it; ++j) {
            // nid: checked ids of tile j + 1.  All shuffles of an iteration come before its loads.
            // Keys that no row sees hold anything: 0.  (Those behind the last row's were not loaded.
            // The test of a key before a window, where its loads are, took 7 to 10 %.)
            if (a.window) {
#pragma unroll
                for (int y = 0; y < 2; ++y)
                    if (!rows_see.one(first(j) + (y ? 32 + (lane & 15) : lane)))
                        num[y] = 0;
            }
            uint32_t by[2];                    // step and middle as they go into the tile
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                float step = __uint_as_float(num[y] << 16), mid = __uint_as_float(num[y] & 0xffff0000u);
                float most = fmaf(8.0f, fabsf(step), fabsf(mid));
                // (so do those of a token that was never stored, seen by its own row: what no written
                // row has, NaN and infinities among it, would reach the tile's other rows)
                if (!(most <= 0x1p120f))
                    step = mid = most = 0.0f;
#pragma unroll
                for (int o = 1; o < 16; o <<= 1)
                    most = fmaxf(most, __shfl_xor_sync(~0u, most, o));
                // 2^e: the largest, no less than any value or 8 of any step, in [2^14, 2^15)
                const int e = max(static_cast<int>(__float_as_uint(most) >> 23) - 127 - 14, -100);
                const float unit = __uint_as_float(static_cast<uint32_t>(127 + e) << 23);
                const float inv = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
                by[y] = pack_half(step * inv, mid * inv);
                if (EXACT && v_side && (y == 0 || (n == 3 && lane < 16)))
                    v_mids[(j & 3) * 128 + 16 * u0 + (y ? 32 : 0) + lane] = fmaf(0.5f, step, mid) * inv;
                if ((lane & 15) == 0 && (y == 0 || (lane == 0 && n == 3))) {
                    const int at = u0 + (y ? 2 : lane >> 4);
                    if (v_side)
                        v_scales[j & 3][at] = make_float2(static_cast<float>(e), share_of(unit));
                    else
                        k_scales[j & 3][at] = unit * mul0;
                }
            }
            uint32_t row_by[3][NL];            // and those of the lane's rows
#pragma unroll
            for (int u = 0; u < 3; ++u)
#pragma unroll
                for (int i = 0; i < NL; ++i)
                    row_by[u][i] = __shfl_sync(~0u, by[u >> 1], 16 * (u & 1) + i * RP + r0);
            uint4 next[3][NL];
            load(next, j + 1, nid);
            after = ask(j + 2);
            __syncwarp();
            if (lane == 0)
                mbar_arrive(bar(SC_FULL + (j & 3)));
            const int st = j & 1;
            if (j >= 2 && ok)
                ok = mbar_park(bar(empty_bar + st), ((j >> 1) - 1) & 1, a.status);
            if (!v_side) {
                // the 16 more dimensions of the lane's keys
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const __half2 both = *reinterpret_cast<const __half2 *>(&by[y]);
                    const int row = 16 * u0 + (y ? 32 + lane : lane);
                    if (y == 0 || (n == 3 && lane < 16))
                        sts128(sbase + S::off_n + row * 128 + (((2 * st) ^ (row & 7)) << 4), half2_bits(__high2half2(both)),
                               half2_bits(__hmul2(__low2half2(both), __float2half2_rn(0.5f))), 0, 0);
                }
            }
            const uint32_t tile = at0 + st * S::tile;
#pragma unroll
            for (int u = 0; u < 3; ++u) {
                if (u == 2 && n == 2)
                    break;
#pragma unroll
                for (int i = 0; i < NL; ++i) {
                    const __half2 both = *reinterpret_cast<const __half2 *>(&row_by[u][i]), step = __low2half2(both);
                    const __half2 add = whole ? __high2half2(both) : __float2half2_rn(-0.0f);
                    const uint32_t word[4] = {v[u][i].x, v[u][i].y, v[u][i].z, v[u][i].w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        uint32_t f[4];
                        codes8_half(word[k], less, step, add, f);
                        sts128(tile + (16 * u + i * RP) * 128 + (sw ^ (16 * k)), f[0], f[1], f[2], f[3]);
                    }
                }
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0)
                mbar_arrive(bar(full_bar + st));
#pragma unroll
            for (int u = 0; u < 3; ++u)
#pragma unroll
                for (int i = 0; i < NL; ++i)
                    v[u][i] = next[u][i];
            nid = check(after);
        }
        if (bad)
            atomicOr(a.status, FKV_ST_RANGE);
    };

    if (FOUR && group >= 2)
        asm volatile("setmaxnreg.dec.sync.aligned.u32 96;");       // (all warps of a group by the same instruction)
    if (FOUR && group >= 2 && warp != 12) {
        // 4-bit codes take more instructions: V's are four warps', K's three of the issuer's
        // group's (units 0 to 2, 3 to 5, 6 and 7 of a tile).  (One place for both: what every
        // warp executes competes for the instruction cache.)
        convert4(group == 2, group == 2 ? 2 * (warp & 3) : 3 * (warp - 13), warp < 15 && group == 3 ? 3 : 2);
    } else if (group == 3) {
        if (!FOUR)
            asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        // ---------------------------------------------------- MMA issuer
        // One elected thread follows the loop: what it waits for, it waits for alone.
        // (K's next tile is waited for before the weights; after the product with V it
        // cost 1 to 3 %.)
        if (warp == 12 && n_it > 0) {
            constexpr uint32_t id_s = idesc_f16_f32(128, 128), id_o = idesc_f16_f32(128, D) | 1u << 16;
            constexpr uint32_t step = S::tile >> 4;
            const uint32_t q_d = static_cast<uint32_t>(sdesc_sw128(sbase + S::off_q));
            const uint32_t k_d = static_cast<uint32_t>(sdesc_sw128(sbase + S::off_k));
            const uint32_t v_d = static_cast<uint32_t>(sdesc_mn_sw128(sbase + S::off_v, S::half));
            const uint32_t v_hi = static_cast<uint32_t>(sdesc_mn_sw128(0, S::half) >> 32);
            bool ok = true;                    // (see the softmax's)
            auto wait = [&](int b, int parity) { ok = ok && mbar_park(bar(b), parity, a.status); };
            auto scores = [&](int w, int j) {
                umma_tile_ss<D>(tmem + 128 * w, q_d + w * step, k_d + (j & 1) * step, id_s);
                if (FOUR)
                    umma_f16(tmem + 128 * w, sdesc_sw128(sbase + S::off_n + 64 + 32 * w), sdesc_sw128(sbase + S::off_n + 32 * (j & 1)), id_s, 1);
                umma_commit(bar(S_FULL + w));
            };
            if (elect_one()) {
                wait(Q_FULL, 0);
                wait(K_FULL, 0);
                tc_fence_after();
                for (int w = n_first > 0 ? 0 : 1; w < groups; ++w)
                    scores(w, 0);
                umma_commit(bar(K_EMPTY));
                for (int j = 0; j < n_it; ++j) {
                    wait(V_FULL + (j & 1), (j >> 1) & 1);
                    if (j + 1 < n_it)
                        wait(K_FULL + ((j + 1) & 1), ((j + 1) >> 1) & 1);
                    for (int w = j < n_first ? 0 : 1; w < groups; ++w) {
                        wait(P_FULL + w, j & 1);
                        tc_fence_after();
                        umma_tile_ts(tmem + 256 + 128 * w, tmem + 128 * w, v_d + (j & 1) * step, id_o, j > 0, v_hi);
                        if (w == groups - 1)
                            umma_commit(bar(V_EMPTY + (j & 1)));
                        if (j + 1 == (w ? n_it : n_first)) {
                            umma_commit(bar(O_FULL + w));
                            continue;
                        }
                        scores(w, j + 1);
                        if (w == groups - 1)
                            umma_commit(bar(K_EMPTY + ((j + 1) & 1)));
                    }
                }
                // every MMA has completed before tensor memory is released
                umma_commit(bar(DRAIN));
                mbar_park(bar(DRAIN), 0, a.status);
            }
            __syncwarp();
        }
    } else if (group == 2) {
        if constexpr (!FOUR) {
            asm volatile("setmaxnreg.dec.sync.aligned.u32 120;");
            // ---------------------------------------------------- codes to fp16 tiles
            // warps 0 and 1 take K's keys 0 .. 63 and 64 .. 127 of a tile, 2 and 3 V's:
            // four units of 16 keys, each of one page
            // A lane moves 16-byte piece c of rows r0, r0 + RP, ...; eight lanes that
            // store together hold four pieces of two rows of different parity, which
            // the swizzle puts on different banks.
            constexpr int RP = 512 / D, NL = 16 / RP;                 // rows at a time, loads a unit
            const int w = warp & 1;
            const int c = D == 128 ? (lane & 3) | (lane >> 1 & 4) : lane & 3;
            const int r0 = D == 128 ? (lane >> 2 & 1) | (lane >> 3 & 2) : lane >> 2;
            // the keys between these are seen by every row
            const int seen_from = a.window ? pb - a.window + 1 : 0;
            const int seen_to = pa < 0 ? 0 : max(a.window ? 0 : q.pre, a.causal ? min(q.len, pa + 1) : q.len);
            const bool v_side = warp & 2;
            const uint8_t *const pool = static_cast<const uint8_t *>(v_side ? a.pool_v : a.pool_k) + h * a.sh + c * 16 + r0 * a.st;
            const float *const scale_of = (v_side ? a.vs : a.ks) + h * a.sch;
            const float mul0 = score_multiplier(a, fabsf(a.scale));
            const int full_bar = v_side ? V_FULL : K_FULL, empty_bar = v_side ? V_EMPTY : K_EMPTY;
            // where the lane's first row's two 16-byte halves go in a tile
            const uint32_t at0 = sbase + (v_side ? S::off_v : S::off_k) + (c >> 2) * S::half + (64 * w + r0) * 128;
            const uint32_t sw = static_cast<uint32_t>((2 * (c & 3)) ^ (r0 & 7)) * 16;
            const int64_t row_step = RP * a.st;
            bool bad = false, ok = true;           // (ok: see the softmax's)
            // Lane u < 4 looks after unit u: its page id (-1: no row sees a key of it)
            // is asked for two tiles ahead and checked a tile later, its scale and the
            // codes one tile ahead, so that nothing here waits for memory.
            auto first = [&](int j) { return tile_at(j) * kTile + 64 * w; };
            struct Page {
                int id;
                bool on;
            };
            auto ask = [&](int j) {
                const int key = first(j) + 16 * lane;
                Page p = {-1, j < n_it && lane < 4 && rows_see.of(key)};
                if (p.on)
                    p.id = a.table[r * a.table_stride + a.div.div(key)];
                return p;
            };
            auto check = [&](const Page &p) {
                if (p.on && (p.id < 0 || p.id >= a.n_blocks)) {
                    bad = true;
                    return 0;
                }
                return p.id;
            };
            auto ask_scale = [&](int id) { return id >= 0 ? scale_of[id * a.scb] : 1.0f; };
            uint4 v[4][NL];
            auto load = [&](int j, int id) {
                // the unit's first row in the pool, from the lane that knows its page
                int64_t from = -1;
                if (id >= 0) {
                    const int key = first(j) + 16 * lane;
                    from = id * a.sb + (key - static_cast<int>(a.div.div(key)) * a.block) * a.st;
                }
                // all of them before the first load: a shuffle behind one waits for it as well
                int64_t at[4];
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    at[u] = __shfl_sync(~0u, from, u);
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const uint8_t *p = pool + at[u];
#pragma unroll
                    for (int i = 0; i < NL; ++i, p += row_step)
                        v[u][i] = at[u] >= 0 ? __ldg(reinterpret_cast<const uint4 *>(p)) : make_uint4(0, 0, 0, 0);
                }
            };
            const Page start = ask(0);
            Page after = ask(1);
            int nid = check(start);
            load(0, nid);
            float scale = ask_scale(nid);
            nid = check(after);
            for (int j = 0; j < n_it; ++j) {
                // nid: checked ids of tile j + 1
                after = ask(j + 2);
                if (lane < 4) {
                    if (v_side) {
                        const float vs = value_scale(scale);
                        v_scales[j & 3][4 * w + lane] = make_float2(lg2(vs), share_of(vs));
                    } else {
                        k_scales[j & 3][4 * w + lane] = scale * mul0;
                    }
                }
                scale = ask_scale(nid);
                __syncwarp();
                if (lane == 0)
                    mbar_arrive(bar(SC_FULL + (j & 3)));
                const int st = j & 1;
                if (j >= 2 && ok)
                    ok = mbar_park(bar(empty_bar + st), ((j >> 1) - 1) & 1, a.status);
                if (FMT == FKV_E4M3 && v_side && (first(j) < seen_from || first(j) + 64 > seen_to)) {
                    // keys that some row does not see hold any bytes, and a weight of zero does
                    // not undo a NaN code
#pragma unroll
                    for (int u = 0; u < 4; ++u)
#pragma unroll
                        for (int i = 0; i < NL; ++i) {
                            v[u][i].x = without_nan(v[u][i].x), v[u][i].y = without_nan(v[u][i].y);
                            v[u][i].z = without_nan(v[u][i].z), v[u][i].w = without_nan(v[u][i].w);
                        }
                }
                const uint32_t tile = at0 + st * S::tile;
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int i = 0; i < NL; ++i) {
                        uint32_t f[8];
                        codes4_half<FOUR ? FKV_E4M3 : FMT>(v[u][i].x, f[0], f[1]);
                        codes4_half<FOUR ? FKV_E4M3 : FMT>(v[u][i].y, f[2], f[3]);
                        codes4_half<FOUR ? FKV_E4M3 : FMT>(v[u][i].z, f[4], f[5]);
                        codes4_half<FOUR ? FKV_E4M3 : FMT>(v[u][i].w, f[6], f[7]);
                        // the row's place in its group of eight turns with i for RP = 4
                        const uint32_t at = tile + (16 * u + i * RP) * 128, x = RP == 4 && (i & 1) ? sw ^ 64 : sw;
                        sts128(at + x, f[0], f[1], f[2], f[3]);
                        sts128(at + (x ^ 16), f[4], f[5], f[6], f[7]);
                    }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0)
                    mbar_arrive(bar(full_bar + st));
                load(j + 1, nid);
                nid = check(after);
            }
            if (bad)
                atomicOr(a.status, FKV_ST_RANGE);
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 160;");
        // ---------------------------------------------------- softmax
        const int w = group, row = row0 + 128 * w + (tid & 127);
        const bool live = row < rows;
        if (w < groups) {
            const int i = live ? static_cast<int>(a.gdiv.div(row)) : 0, u = live ? row - i * a.G : 0;
            const int64_t tok = q.tok0 + i, head = h * a.G + u;
            Row st;
            st.m = live ? -INFINITY : 0.0f, st.l = 0.0f, st.down = 1.0f, st.mid = 0.0f;
            st.p = q.p0 + i;
            const RowMask mask(a, q, st.p, live);
            st.hi = mask.hi, st.from = mask.from, st.pre = mask.pre;
            st.slope = a.slopes && live ? a.slopes[head] * kLog2e : 0.0f;
            // The warp's 32 query rows as fp16 (a negative scale turns their sign), LR lanes
            // a row: with a row a lane each access would touch 32 lines, 2000 cycles a
            // block for 64 dimensions.
            const int first = row0 + 128 * w + 32 * (warp & 3);
            const uint32_t q_tile = sbase + S::off_q + w * S::tile + 32 * (warp & 3) * 128;
            // 16-byte piece k of row r of the warp's in a tile of 128-byte rows
            auto piece = [&](int r, int k) { return q_tile + (k >> 3) * S::half + r * 128 + (((k & 7) ^ (r & 7)) << 4); };
            {
                constexpr int LR = D / 8, RI = 32 / LR;                  // rows at a time
                // (with 4-bit keys rows of either type are scaled, and to less, so that fp16
                // holds their sums: elements below 2^-21 of the largest are rounded to 2^-32 of it)
                constexpr int TOP = FOUR ? 7 : 14;
                float all = 0.0f;                                        // the lane's row's sum
                const int c = lane % LR, rr = lane / LR;
                uint4 v[LR];
#pragma unroll
                for (int k = 0; k < LR; ++k) {
                    const int x = first + k * RI + rr;
                    v[k] = make_uint4(0, 0, 0, 0);
                    if (x < rows) {
                        const int xi = static_cast<int>(a.gdiv.div(x));
                        const T *src = static_cast<const T *>(a.q) + (q.tok0 + xi) * a.q_tok + (h * a.G + x - xi * a.G) * a.q_head;
                        v[k] = reinterpret_cast<const uint4 *>(src)[c];
                    }
                }
#pragma unroll
                for (int k = 0; k < LR; ++k) {
                    uint32_t y[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
                    if (!FOUR && std::is_same<T, __half>::value) {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            y[e] ^= a.scale < 0.0f ? 0x80008000u : 0u;
                    } else if (std::is_same<T, __half>::value) {
                        float m = 0.0f;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float2 z = __half22float2(*reinterpret_cast<const __half2 *>(&y[e]));
                            m = fmaxf(m, fmaxf(fabsf(z.x), fabsf(z.y)));
                        }
#pragma unroll
                        for (int o = 1; o < LR; o *= 2)
                            m = fmaxf(m, __shfl_xor_sync(~0u, m, o));
                        const int e2 = max(static_cast<int>(__float_as_uint(m) >> 23) - 127, -100);
                        float up = __uint_as_float(static_cast<uint32_t>(127 + TOP - e2) << 23);
                        const float down = __uint_as_float(static_cast<uint32_t>(127 - TOP + e2) << 23);
                        const float mine = __shfl_sync(~0u, down, lane % RI * LR);
                        if (lane / RI == k)
                            st.down = mine;
                        up = a.scale < 0.0f ? -up : up;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float2 z = __half22float2(*reinterpret_cast<const __half2 *>(&y[e]));
                            y[e] = pack_half(z.x * up, z.y * up);
                        }
                    } else {
                        // brought to [2^14, 2^15) by a power of two (see attend.cu)
                        uint32_t m = 0;
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            asm("max.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(y[e] & 0x7fff7fffu));
                        m = max(m & 0xffffu, m >> 16);
#pragma unroll
                        for (int o = 1; o < LR; o *= 2)
                            m = max(m, __shfl_xor_sync(~0u, m, o));
                        const int e2 = max(static_cast<int>(m >> 7) - 127, -100);
                        float up = __uint_as_float(static_cast<uint32_t>(127 + TOP - e2) << 23);
                        const float down = __uint_as_float(static_cast<uint32_t>(127 - TOP + e2) << 23);
                        const float mine = __shfl_sync(~0u, down, lane % RI * LR);
                        if (lane / RI == k)
                            st.down = mine;
                        up = a.scale < 0.0f ? -up : up;
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            y[e] = pack_half(__uint_as_float(y[e] << 16) * up, __uint_as_float(y[e] & 0xffff0000u) * up);
                    }
                    if (FOUR) {
                        // the row's sum, and the order of the codes
                        float sum = 0.0f;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float2 z = __half22float2(*reinterpret_cast<const __half2 *>(&y[e]));
                            sum += z.x + z.y;
                        }
#pragma unroll
                        for (int o = 1; o < LR; o *= 2)
                            sum += __shfl_xor_sync(~0u, sum, o);
                        const float mine = __shfl_sync(~0u, sum, lane % RI * LR);
                        if (lane / RI == k)
                            all = mine;
                        sts128(piece(k * RI + rr, c), __byte_perm(y[0], y[2], 0x5410), __byte_perm(y[0], y[2], 0x7632),
                               __byte_perm(y[1], y[3], 0x5410), __byte_perm(y[1], y[3], 0x7632));
                    } else {
                        sts128(piece(k * RI + rr, c), y[0], y[1], y[2], y[3]);
                    }
                }
                if (FOUR) {
                    const float hi = __half2float(__float2half_rn(all));
                    const uint32_t both = pack_half(hi, all - hi);
                    const int rl = 32 * (warp & 3) + lane;
                    sts128(sbase + S::off_n + rl * 128 + (((4 + 2 * w) ^ (rl & 7)) << 4), both, both, 0, 0);
                }
                fence_proxy_async_smem();
                mbar_arrive(bar(Q_FULL));
            }
            // the group's own range of positions, for tiles that need no mask
            const int ga = q.p0 + static_cast<int>(a.gdiv.div(row0 + 128 * w));
            const int gb = q.p0 + static_cast<int>(a.gdiv.div(min(row0 + 128 * w + 128, rows) - 1));
            const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
            const uint32_t s_t = tmem + 128 * w + lanes, o_t = tmem + 256 + 128 * w + lanes;
            // A thread that gives up waits no more but goes on with what it finds, to the
            // loop's end (the call has failed and says so): one that left would be waited
            // for by its warp, whose next step is for all its threads, for ever.
            bool ok = true;
            const int n_own = w ? n_it : n_first;
            for (int j = 0; j < n_own; ++j) {
                ok = ok && mbar_park(bar(SC_FULL + (j & 3)), (j >> 2) & 1, a.status);
                const int key = tile_at(j) * kTile;
                const float *const km = k_scales[j & 3];
                const float2 *const vm = v_scales[j & 3];
                const float4 *const mids = reinterpret_cast<const float4 *>(v_mids + (j & 3) * 128);
                const bool full = all_see(a, q, ga, gb, key, key + kTile);
                // before the scores are there: the pages' multipliers
                float km_r[8], vo_r[8];
#pragma unroll
                for (int n = 0; n < 8; ++n)
                    km_r[n] = km[n] * st.down, vo_r[n] = vm[n].x;
                ok = ok && mbar_park(bar(S_FULL + w), j & 1, a.status);
                tc_fence_after();
                // the visible ones of 32 keys as bits: ranges meet as words, and a score's
                // test is one bit (its three comparisons, short cuts and all, took 80
                // cycles a score)
                auto seen = [&](int j0) {
                    return (below(st.hi - j0) & (~below(st.from - j0) | below(a.sinks - j0))) | below(st.pre - j0);
                };
                // products to scores in base 2 where a cap or a bias is between them
                auto general = [&](float *s, int half, const float *mul, const float *off) {
                    if (SCORES == SCORES_LARGE_CAP) {
                        // mostly no score is near the cap, and the series is all there is to do
                        float most = 0.0f;
#pragma unroll
                        for (int e = 0; e < 64; ++e) {
                            s[e] *= mul[e / 16];
                            most = fmaxf(most, fabsf(s[e]));
                        }
                        if (__any_sync(~0u, !(most * a.cap_inv < 0.5f))) {
#pragma unroll
                            for (int e = 0; e < 64; ++e)
                                s[e] = capped(a, s[e]) + off[e / 16];
                        } else {
#pragma unroll
                            for (int e = 0; e < 64; ++e)
                                s[e] = capped_near(a, s[e]) + off[e / 16];
                        }
                    } else if (a.softcap > 0.0f) {
                        const float cap = a.cap2;
#pragma unroll
                        for (int e = 0; e < 64; ++e)
                            s[e] = fmaf(-2.0f * cap, __fdividef(1.0f, 1.0f + ex2(s[e] * mul[e / 16])), cap + off[e / 16]);
                    } else {
#pragma unroll
                        for (int e = 0; e < 64; e += 2)
                            fma2(s[e], s[e + 1], s[e], s[e + 1], mul[e / 16], off[e / 16]);
                    }
                    if (a.slopes) {
                        const float at = static_cast<float>(key + 64 * half - st.p);
#pragma unroll
                        for (int e = 0; e < 64; ++e)
                            s[e] = fmaf(st.slope, at + static_cast<float>(e), s[e]);
                    }
                };
                // A tile whose rows have their reference: two halves of 64 columns, the
                // second's products on their way while the first's weights are stored.
                int k = 0, again = j == 0;
                if (j > 0) {
                    float s[64], sum[4], mid[2];
                    uint32_t p[32];
                    auto evaluate = [&](int half) {
                        mid[0] = mid[1] = 0.0f;
#pragma unroll
                        for (int n = 0; n < 4; ++n) {
                            float sx = 0.0f, sy = 0.0f;
                            const float mul = GEN ? 1.0f : half ? km_r[4 + n] : km_r[n], o = (GEN ? 0.0f : half ? vo_r[4 + n] : vo_r[n]) - st.m;
#pragma unroll
                            for (int e = 16 * n; e < 16 * n + 16; e += 2) {
                                float y0, y1;
                                fma2(y0, y1, s[e], s[e + 1], mul, o);
                                y0 = ex2(y0), y1 = ex2(y1);
                                add2(sx, sy, y0, y1);
                                if (EXACT) {
                                    const float4 h = mids[16 * half + e / 4];
                                    fma2_each(mid[0], mid[1], y0, y1, e % 4 ? h.z : h.x, e % 4 ? h.w : h.y, mid[0], mid[1]);
                                }
                                p[e >> 1] = pack_half(y0, y1);
                            }
                            sum[n] = sx + sy;
                        }
                        // (not <=: a sum that is no number is looked at as well)
                        return __any_sync(~0u, !((sum[0] + sum[1]) + (sum[2] + sum[3]) <= kMostSum) ||
                                                   st.m == -INFINITY);
                    };
                    // a masked product is -infinity (times a multiplier of zero no number,
                    // which is looked at below)
                    auto hide = [&](int half) {
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            const uint32_t vis = seen(key + 64 * half + 32 * x);
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                s[32 * x + e] = vis >> e & 1 ? s[32 * x + e] : -INFINITY;
                        }
                    };
                    tmem_ld32(s_t, s);
                    tmem_ld32(s_t + 32, s + 32);
                    tmem_wait_ld(s);
                    tmem_wait_ld(s + 32);
                    if (GEN)
                        general(s, 0, km_r, vo_r);
                    if (!full)
                        hide(0);
                    again = evaluate(0);
                    if (!again) {
                        tmem_ld32(s_t + 64, s);
                        tmem_ld32(s_t + 96, s + 32);
#pragma unroll
                        for (int n = 0; n < 4; ++n)
                            st.l = fmaf(sum[n], vm[n].y, st.l);
                        st.mid += mid[0] + mid[1];
                        // fp16 pairs in the tile's first columns, which have been read
                        tmem_st16(s_t, p);
                        tmem_st16(s_t + 16, p + 16);
                        tmem_wait_ld(s);
                        tmem_wait_ld(s + 32);
                        k = 1;
                        if (GEN)
                            general(s, 1, km_r + 4, vo_r + 4);
                        if (!full)
                            hide(1);
                        again = evaluate(1);
                        if (!again) {
#pragma unroll
                            for (int n = 0; n < 4; ++n)
                                st.l = fmaf(sum[n], vm[4 + n].y, st.l);
                            st.mid += mid[0] + mid[1];
                            tmem_st16(s_t + 32, p);
                            tmem_st16(s_t + 48, p + 16);
                            k = 2;
                        }
                        tmem_wait_st();
                    }
                }
                // Any other tile: a half at a time, a second time where the reference has
                // to move first.
#pragma unroll 1
                while (k < 2) {
                    float s[64];
                    tmem_ld32(s_t + 64 * k, s);
                    tmem_ld32(s_t + 64 * k + 32, s + 32);
                    tmem_wait_ld(s);
                    tmem_wait_ld(s + 32);
                    float mul[4], off[4];
#pragma unroll
                    for (int n = 0; n < 4; ++n) {
                        mul[n] = km[4 * k + n] * st.down;
                        off[n] = vm[4 * k + n].x;
                    }
                    if (GEN || !full) {
                        if (GEN) {
                            general(s, k, mul, off);
                        } else {
#pragma unroll
                            for (int e = 0; e < 64; e += 2)
                                fma2(s[e], s[e + 1], s[e], s[e + 1], mul[e / 16], off[e / 16]);
                        }
                        if (!full) {
#pragma unroll
                            for (int x = 0; x < 2; ++x) {
                                const uint32_t vis = seen(key + 64 * k + 32 * x);
#pragma unroll
                                for (int e = 0; e < 32; ++e)
                                    s[32 * x + e] = vis >> e & 1 ? s[32 * x + e] : -INFINITY;
                            }
                        }
#pragma unroll
                        for (int n = 0; n < 4; ++n)
                            mul[n] = 1.0f, off[n] = 0.0f;
                    }
                    if (again) {
                        // A score's weight is 2^(score - m); m an integer.  All of the
                        // warp's rows move up to what they have seen: one at a time they
                        // would each bring the warp here.
                        float mx = -INFINITY;
#pragma unroll
                        for (int e = 0; e < 64; ++e)
                            mx = fmaxf(mx, fmaf(s[e], mul[e / 16], off[e / 16]));
                        const float to = fmaxf(st.m, mx > -INFINITY ? ceilf(mx) - kPBits : st.m);
                        const float f = to == st.m ? 1.0f : ex2(st.m - to);
                        // (the sum in two halves: counted up to 2^80 a weight, it outlasts
                        // factors below float32's least)
                        const float half = to == st.m ? 1.0f : ex2(0.5f * (st.m - to));
                        st.m = to;
                        st.l = st.l * half * half;
                        st.mid *= f;
                        // the products so far are done: their commit came before this tile's scores'
                        if (j > 0) {
#pragma unroll 1
                            for (int c = 0; c < D; c += 16) {
                                uint32_t o[16];
                                tmem_ld16(o_t + c, o);
#pragma unroll
                                for (int e = 0; e < 16; ++e)
                                    o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                                tmem_st16(o_t + c, o);
                            }
                        }
                        if (k > 0) {
                            // in fp32: a factor below fp16's least, 2^-24, still leaves weights
                            // of up to 2^15 something
#pragma unroll 1
                            for (int c = 0; c < 32; c += 16) {
                                uint32_t o[16];
                                tmem_ld16(s_t + c, o);
#pragma unroll
                                for (int e = 0; e < 16; ++e) {
                                    const float2 y = __half22float2(*reinterpret_cast<const __half2 *>(&o[e]));
                                    o[e] = pack_half(y.x * f, y.y * f);
                                }
                                tmem_st16(s_t + c, o);
                            }
                        }
                        tmem_wait_st();
                    }
                    const float base = again && st.m == -INFINITY ? 0.0f : st.m;
                    uint32_t p[32];
                    float sum[4], mid[2] = {0.0f, 0.0f};
#pragma unroll
                    for (int n = 0; n < 4; ++n) {
                        float sx = 0.0f, sy = 0.0f;
                        const float o = off[n] - base;
#pragma unroll
                        for (int e = 16 * n; e < 16 * n + 16; e += 2) {
                            float y0, y1;
                            fma2(y0, y1, s[e], s[e + 1], mul[n], o);
                            y0 = ex2(y0), y1 = ex2(y1);
                            add2(sx, sy, y0, y1);
                            if (EXACT) {
                                const float4 h = mids[16 * k + e / 4];
                                fma2_each(mid[0], mid[1], y0, y1, e % 4 ? h.z : h.x, e % 4 ? h.w : h.y, mid[0], mid[1]);
                            }
                            p[e >> 1] = pack_half(y0, y1);
                        }
                        sum[n] = sx + sy;
                    }
                    // (not <=: a sum that is no number is looked at as well)
                    if (!again && __any_sync(~0u, !((sum[0] + sum[1]) + (sum[2] + sum[3]) <= kMostSum) ||
                                                      st.m == -INFINITY)) {
                        again = 1;
                        continue;
                    }
#pragma unroll
                    for (int n = 0; n < 4; ++n)
                        st.l = fmaf(sum[n], vm[4 * k + n].y, st.l);
                    st.mid += mid[0] + mid[1];
                    // fp16 pairs in the tile's first columns, which have been read
                    tmem_st16(s_t + 32 * k, p);
                    tmem_st16(s_t + 32 * k + 16, p + 16);
                    tmem_wait_st();
                    ++k;
                    again = 0;
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0)
                    mbar_arrive(bar(P_FULL + w));
            }
            if (n_own > 0 && ok)
                mbar_park(bar(O_FULL + w), 0, a.status);
            __syncwarp();
            tc_fence_after();
            const float inv = st.l != 0.0f ? kRef / st.l : 0.0f;
            const float lse2 = st.l != 0.0f ? st.m + log2f(st.l) - kLog2Ref : -INFINITY;
            const int64_t flat = tok * (a.H * a.G) + head, at = split * a.T * (a.H * a.G) + flat;
            // Rows meet in the group's query tile, which no product reads any more, 128
            // bytes of each at a time, and eight lanes write a row's.
            auto flush = [&](int chunk) {
                __syncwarp();
#pragma unroll 2
                for (int k = 0; k < 8; ++k) {
                    const int rl = 4 * k + (lane >> 3), x = first + rl;
                    if (x >= rows)
                        continue;
                    const int xi = static_cast<int>(a.gdiv.div(x));
                    const int64_t xt = q.tok0 + xi, xh = h * a.G + x - xi * a.G;
                    uint8_t *dst = a.splits == 1
                                       ? reinterpret_cast<uint8_t *>(static_cast<T *>(a.out) + xt * a.o_tok + xh * a.o_head)
                                       : reinterpret_cast<uint8_t *>(a.ws_o + ((split * a.T + xt) * (a.H * a.G) + xh) * D);
                    *reinterpret_cast<uint4 *>(dst + chunk * 128 + (lane & 7) * 16) =
                        *reinterpret_cast<const uint4 *>(raw + (piece(rl, lane & 7) - smem_u32(raw)));
                }
                __syncwarp();
            };
#pragma unroll 1
            for (int k = 0; k < D / 32; ++k) {
                float o[32];
                tmem_ld32(o_t + 32 * k, o);
                tmem_wait_ld(o);
                // a row that saw nothing has no products either: tensor memory holds anything
#pragma unroll
                for (int e = 0; e < 32; ++e)
                    o[e] = st.l != 0.0f ? (EXACT ? o[e] + st.mid : o[e]) * inv : 0.0f;
                // dimension e of the 32 (4-bit pages: see the codes' order)
                auto dim = [&](int e) { return FOUR ? o[(e & ~7) | (e << 1 & 6) | (e >> 2 & 1)] : o[e]; };
                if (a.splits == 1) {
#pragma unroll
                    for (int e = 0; e < 32; e += 8) {
                        T y[8];
#pragma unroll
                        for (int f = 0; f < 8; ++f)
                            y[f] = from_float<T>(dim(e + f));
                        const uint4 z = *reinterpret_cast<const uint4 *>(y);
                        sts128(piece(lane, 4 * (k & 1) + e / 8), z.x, z.y, z.z, z.w);
                    }
                    if (k & 1)
                        flush(k >> 1);
                } else {
#pragma unroll
                    for (int e = 0; e < 32; e += 4)
                        sts128(piece(lane, e / 4), __float_as_uint(dim(e)), __float_as_uint(dim(e + 1)), __float_as_uint(dim(e + 2)),
                               __float_as_uint(dim(e + 3)));
                    flush(k);
                }
            }
            if (live) {
                if (a.splits > 1)
                    a.ws_lse[at] = lse2;
                else if (a.lse)
                    a.lse[flat] = lse2 / kLog2e;
            }
            tc_fence_before();
        }
    }
    __syncthreads();
    if (warp == 12) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

template <int D, int FMT, typename T, int SCORES> cudaError_t prompt_as(const fkv_ctx *ctx, const AttendArgs &a, cudaStream_t st)
{
    constexpr int smem = PromptShape<D>::smem(FMT);
    const void *fn = reinterpret_cast<const void *>(k_attend_prompt<D, FMT, T, SCORES>);
    const cudaError_t e = kernel_use(ctx, fn, kThreads, smem, nullptr);
    if (e != cudaSuccess)
        return e;
    const unsigned grid = static_cast<unsigned>(static_cast<int64_t>(a.row_tiles) * a.n_req * a.splits * a.H);
    k_attend_prompt<D, FMT, T, SCORES><<<grid, kThreads, smem, st>>>(a);
    return cudaGetLastError();
}

template <int D, int FMT, typename T> cudaError_t prompt_t(const fkv_ctx *ctx, const AttendArgs &a, cudaStream_t st)
{
    if (a.softcap > kPlainCap)
        return prompt_as<D, FMT, T, SCORES_LARGE_CAP>(ctx, a, st);
    return a.softcap > 0.0f || a.slopes ? prompt_as<D, FMT, T, SCORES_GENERAL>(ctx, a, st)
                                        : prompt_as<D, FMT, T, SCORES_PLAIN>(ctx, a, st);
}

template <int D, int FMT> cudaError_t prompt_dt(const fkv_ctx *ctx, const AttendArgs &a, int dtype, cudaStream_t st)
{
    return dtype == FKV_F16 ? prompt_t<D, FMT, __half>(ctx, a, st) : prompt_t<D, FMT, __nv_bfloat16>(ctx, a, st);
}

}  // namespace

// The build compiles this file twice, for 8-bit and for 4-bit pages.
#ifndef FKV_PAGES_4BIT
int prompt_rows() { return kRows; }

cudaError_t launch_attend_prompt(const fkv_ctx *ctx, const AttendArgs &a, int dim, int format, int dtype, cudaStream_t st)
{
    if (dim == 64)
        return format == FKV_INT8 ? prompt_dt<64, FKV_INT8>(ctx, a, dtype, st) : prompt_dt<64, FKV_E4M3>(ctx, a, dtype, st);
    return format == FKV_INT8 ? prompt_dt<128, FKV_INT8>(ctx, a, dtype, st) : prompt_dt<128, FKV_E4M3>(ctx, a, dtype, st);
}
#else
cudaError_t launch_attend_prompt4(const fkv_ctx *ctx, const AttendArgs &a, int dim, int dtype, cudaStream_t st)
{
    return dim == 64 ? prompt_dt<64, FKV_UINT4>(ctx, a, dtype, st) : prompt_dt<128, FKV_UINT4>(ctx, a, dtype, st);
}
#endif
