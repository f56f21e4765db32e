// Attention over 4-bit pages for a few rows a KV head (attend.cu has the mathematics
// of the 8-bit ones and the plan).
//
// Key j is mid_j + (c_j - 7.5) step_j and value j mid'_j + (c'_j - 7.5) step'_j, with
// numbers of their own for every row of a page.  So
//     q.k_j = step_j (q.c_j - 7.5 sum q) + mid_j sum q,
// two multiplications and additions a score behind the product of the query with whole
// numbers, which starts from -7.5 sum q; and with
//     y_j = x_j log2 e + log2 step'_j,   P_j = 2^(y_j - m + 8),   m >= max y_j - 7
// the row's output is
//     (sum P_j (c'_j - 7.5) + sum P_j mid'_j / step'_j) / sum P_j / step'_j,
// the first sum on the tensor cores with P rounded to fp16 (as for 8-bit pages), the
// others of unrounded weights in fp32.  sum P_j 7.5, of the rounded weights as the
// product with c' has them, is one more row of that product, of ones.
//
// A code needs no conversion: as the low four bits of an fp16 number it is the
// subnormal c 2^-24, and one place to the left c 2^-20.  A word of eight codes is four
// operands of two after four masks and a shift; the factor 16 between neighbours is
// taken out of the query for K, exactly but for elements of it below 2^-24 of its largest
// (rounded to 2^-35 of that), and of the output for V.
//
// Half of the bytes of 8-bit pages bring the same work: what bounds these kernels is no longer
// bytes alone.  8 heads of 128, 4 rows each: 64 sequences of 16-32k positions, 311 us, 5.6 TB/s,
// 84 % of a copy's.  Steps (each call timed by itself, 10 us more): 481 us; 64 keys an
// iteration, scores without branches in their loop 404; loads of whole pages' units together
// 380; a warp's number uniform 369; four operations a half word of V, no branch a unit 349;
// two-wide arithmetic 344; V by transposed loads 328; the reference moved only where a weight
// asks for it 321.  One sequence of 131k with a cap 36 us, 3.9 TB/s (two launches' starts and
// ends, 12 us of it); up to 28 rows, 24 sequences, a window of 4,096 and a bias 61 us.  Not
// kept: w >> 8 on the multipliers (403 against 369); four blocks of 128 threads an SM with 32
// keys an iteration (425).
#include "attend_step.cuh"

using namespace fkvd;

namespace {

// As k_attend_step: four warps, each with every fourth group of keys, a ring of its
// own filled by TMA and a softmax of its own; keys are the rows of the first
// product, dimensions those of the second, query rows their 8 columns.  A group is 64
// keys: with 32 what an iteration costs beside its keys came twice (8 rows 418 us instead
// of 369, up to 28 rows with a window 89 instead of 83).
template <int D, int NT> struct Step4Shape {
    static constexpr int keys = kStep4Keys, units = keys / 16;
    static constexpr int stages = D == 128 ? 2 : 3;
    static constexpr int unit = 8 * D, stage = 2 * units * unit;                // 16 keys' codes; a group's
    static constexpr int codes = 4 * stages * stage, ring = codes + 4 * stages * 2 * units * 64;   // with their numbers
    static constexpr int q = NT > 1 ? NT * (D / 16) * 256 : 0;  // the query operands, [column tile][step][lane]
    static constexpr int nums = 4 * keys * 20;                  // a warp's keys' numbers
    static constexpr int ml = 4 * 2 * 8 * NT * 4;
    static constexpr int smem = ring + q + nums + ml + 1024;
};

// Contiguous bytes into shared memory, 16-byte aligned and a multiple of 16 of them.
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, int bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
                 "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(bar)
                 : "memory");
}

// Eight codes as four fp16 pairs: (c0, c4) and (c2, c6) times 2^-24, (c1, c5) and
// (c3, c7) times 2^-20.
__device__ __forceinline__ void codes8_pairs(uint32_t w, uint32_t *f)
{
    const uint32_t x = w >> 8;
    f[0] = w & 0x000f000fu, f[1] = w & 0x00f000f0u;
    f[2] = x & 0x000f000fu, f[3] = x & 0x00f000f0u;
}

// Four codes each of two values, x = (c0 c1 c2 c3, c0' ..): (c0, c0'), (c2, c2') times 2^-24,
// and (c0 + 16 c1, ..), (c2 + 16 c3, ..): an operation less, and what the even dimension
// adds to the odd one's sum is taken off at the end.
__device__ __forceinline__ void codes4_pairs(uint32_t x, uint32_t *f)
{
    const uint32_t y = __byte_perm(x, 0, 0x4341);
    f[0] = x & 0x000f000fu, f[1] = x & 0x00ff00ffu;
    f[2] = y & 0x000f000fu, f[3] = y;
}

// Four 8 x 8 matrices of 16-bit elements from rows of 16 bytes (a lane's address is one of
// eight rows of one of them), transposed: a lane has elements (2t, gid) and (2t + 1, gid).
__device__ __forceinline__ void ldmatrix4_trans(uint32_t *r, uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr));
}

// D = A B + C.
__device__ __forceinline__ void mma16816_from(float *d, const uint32_t *a, uint32_t b0, uint32_t b1, float c0, float c1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%10,%11};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c0), "f"(c1));
}

template <int D, typename T, int NT>
__global__ void __launch_bounds__(128, step4_blocks(NT))
    k_attend_step4(const AttendArgs a, const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv)
{
    using S = Step4Shape<D, NT>;
    constexpr int ST = S::stages, U = S::units, KW = S::keys, PT = kTile / KW, W = D / 32, MO = D / 16, R = 8 * NT;
    extern __shared__ uint8_t raw[];
    __shared__ __align__(8) uint64_t bars[4 * ST];
    __shared__ Seen rows_see[4];                 // a warp's own: registers are short
    // (the same for all of a warp as far as the compiler can see: addresses and loop bounds
    // are uniform then)
    const int tid = threadIdx.x, warp = __shfl_sync(~0u, tid >> 5, 0), lane = tid & 31, gid = lane >> 2, t = lane & 3;
    const uint32_t sbase = (smem_u32(raw) + 1023) & ~1023u;
    uint8_t *const base = raw + (sbase - smem_u32(raw));
    uint2 *const q_s = reinterpret_cast<uint2 *>(base + S::ring);
    // a warp's keys: K's step and middle times 2^11, log2 of V's step; what a weight counts, and times V's middle
    float4 *const keys_s = reinterpret_cast<float4 *>(base + S::ring + S::q) + KW * warp;
    float *const mids_s = reinterpret_cast<float *>(base + S::ring + S::q + 4 * KW * 16) + KW * warp;
    typedef float RowPair[2][R];                 // a warp's maxima and sums
    RowPair *const ml = reinterpret_cast<RowPair *>(base + S::ring + S::q + S::nums);

    const int h = blockIdx.y;
    const int split = blockIdx.x % a.splits, rr = blockIdx.x / a.splits;
    const int rt = rr % a.row_tiles, r = rr / a.row_tiles;
    Request q;
    if (!q.load(a, r)) {
        if (tid == 0)
            atomicOr(a.status, FKV_ST_RANGE);
        return;
    }
    const int rows = q.nq * a.G, row0 = rt * R;
    if (row0 >= rows)
        return;
    const int ia = static_cast<int>(a.gdiv.div(row0)), ib = static_cast<int>(a.gdiv.div(min(row0 + R - 1, rows - 1)));
    const int pa = q.p0 + ia, pb = q.p0 + ib;
    const Tiles tiles(a, q, pa, pb);
    const int i0 = split * a.chunk, i1 = min(tiles.n, i0 + a.chunk);
    // the share's groups of keys, but for those behind all that any row sees; a warp's are
    // every fourth (a bias: from the last one back, see k_attend_step)
    auto group_at = [&](int g) { return tiles.at(i0 + (g >> PT / 2)) * kTile + (g & (PT - 1)) * KW; };
    int groups = max(0, i1 - i0) * PT;
    while (groups > 0 && group_at(groups - 1) >= tiles.lim)
        --groups;
    const int n_it = (groups - warp + 3) >> 2;   // 0 or less: none
    const bool back = a.slopes != nullptr;
    // what every row sees: positions up to first_end, and from begin to last_end
    const int last_end = pa < 0 ? 0 : a.causal ? min(q.len, pa + 1) : q.len, begin = a.window ? pb - a.window + 1 : 0;
    const int first_end = pa < 0 ? 0 : max(q.pre, a.window ? min(a.sinks, last_end) : 0);
    auto first_key = [&](int it) { return group_at(back ? groups - 1 - 4 * it - warp : 4 * it + warp); };

    const uint32_t ring = sbase + warp * ST * S::stage, nums = sbase + S::codes + warp * ST * (2 * U * 64), bar0 = smem_u32(bars) + warp * ST * 8;
    if (lane == 0) {
        rows_see[warp] = tiles.seen;
        for (int s = 0; s < ST; ++s)
            mbar_init(bar0 + 8 * s, 1);
        fence_mbar_init();
    }
    __syncwarp();

    // A lane looks up the page of one of the 32 units (16 keys) of 32 / U iterations, a
    // batch of iterations ahead, if any row sees one of its keys.
    constexpr int BI = 32 / U;
    bool bad = false;
    struct Unit {
        int id;
        unsigned all;                  // which of the 32 units are looked at
    };
    auto key_of = [&](int batch) { return first_key(batch * BI + lane / U) + (lane & (U - 1)) * 16; };
    auto on = [&](int batch) { return batch * BI + lane / U < n_it && rows_see[warp].of(key_of(batch)); };
    auto ask = [&](int batch) { return on(batch) ? a.table[r * a.table_stride + a.div.div(key_of(batch))] : 0; };
    auto check = [&](int batch, int id) {
        const bool mine = on(batch);
        Unit u = {0, __ballot_sync(~0u, mine)};
        if (mine) {
            if (id < 0 || id >= a.n_blocks)
                bad = true;
            else
                u.id = id;
        }
        return u;
    };
    Unit cur = check(0, ask(0)), nxt = check(1, ask(1));
    int nid = ask(2);
    auto units_of = [&](const Unit &u, unsigned it) { return u.all >> ((it & (BI - 1)) * U) & ((1u << U) - 1); };
    // Units are loaded as many together as pages hold whole ones of (2^box): a load takes some
    // 15 instructions, as its operands are the warp's.
    const int pieces = U >> a.box;
    auto issue = [&](unsigned it, unsigned batch) {
        const bool now = it / BI == batch;
        const unsigned units = units_of(now ? cur : nxt, it);
        const int x = lane & (pieces - 1), u = x << a.box, what = lane >> (31 - __clz(pieces));
        // (whichever of a piece's units any row sees has its page)
        const unsigned mine = units >> u & ((1u << (1 << a.box)) - 1);
        const int64_t id = __shfl_sync(~0u, now ? cur.id : nxt.id, (it & (BI - 1)) * U + u + (mine ? __ffs(mine) - 1 : 0));
        const int key = first_key(it) + u * 16, off = key - static_cast<int>(a.div.div(key)) * a.block;
        const uint32_t bar = bar0 + 8 * (it % ST), slot = it % ST;
        const unsigned heads = __ballot_sync(~0u, lane < pieces && mine);
        // (without any the arrival alone completes the phase)
        if (lane == 0)
            mbar_arrive_expect_tx(bar, __popc(heads) * 2 * (S::unit + 64) << a.box);
        __syncwarp();
        // `pieces` lanes each: codes of K, of V, their numbers
        if (what < 4 && mine) {
            if (what < 2)
                tma_load_4d(ring + slot * S::stage + (what * U + u) * S::unit, what ? &mv : &mk, 0, off, h, static_cast<int>(id), bar);
            else
                bulk_load(nums + slot * (2 * U * 64) + ((what - 2) * U + u) * 64, (what < 3 ? a.ks : a.vs) + id * a.scb + h * a.sch + off,
                          64 << a.box, bar);
        }
        __syncwarp();
    };
    for (int it = 0; it < min(ST - 1, n_it); ++it)
        issue(it, 0);

    // The query rows as fp16 operands: lane t's steps take D / 4 consecutive dimensions
    // of row gid, brought to [2^14, 2^15) by a power of two, eight at a time in the order
    // of codes8_pairs.
    const float mul0 = score_multiplier(a, a.scale);
    uint32_t qf[NT > 1 ? 1 : 2 * W][2];
    float rowmul[NT][2], rowsum[NT][2], start[NT][2], slope[NT][2];
    int prow[NT][2], hi[NT][2], from[NT][2], pre[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int row = row0 + 8 * n + gid;
        const bool live = row < rows;
        const int i = live ? static_cast<int>(a.gdiv.div(row)) : 0, u = live ? row - i * a.G : 0;
        const T *src = static_cast<const T *>(a.q) + (q.tok0 + i) * a.q_tok + (h * a.G + u) * a.q_head + t * (D / 4);
        float x[W][8];
        float amax = 0.0f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            uint4 v = make_uint4(0, 0, 0, 0);
            if (live)
                v = reinterpret_cast<const uint4 *>(src)[w];
            const T *y = reinterpret_cast<const T *>(&v);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                x[w][k] = static_cast<float>(y[k]);
                amax = fmaxf(amax, fabsf(x[w][k]));
            }
        }
        amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, 1));
        amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, 2));
        const int e = max(static_cast<int>(__float_as_uint(amax) >> 23) - 127, -100);
        const float up = __uint_as_float(static_cast<uint32_t>(127 + 14 - e) << 23);
        const float down = __uint_as_float(static_cast<uint32_t>(127 - 14 + e) << 23);
        float sum = 0.0f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                x[w][k] *= up;
                sum += x[w][k];
            }
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const uint32_t f0 = pack_half(x[w][2 * s], x[w][2 * s + 4]);
                const uint32_t f1 = pack_half(x[w][2 * s + 1] * 0.0625f, x[w][2 * s + 5] * 0.0625f);
                if (NT > 1) {
                    if (warp == n % 4)
                        q_s[(n * 2 * W + 2 * w + s) * 32 + lane] = make_uint2(f0, f1);
                } else {
                    qf[2 * w + s][0] = f0, qf[2 * w + s][1] = f1;
                }
            }
        }
        sum += __shfl_xor_sync(~0u, sum, 1);
        sum += __shfl_xor_sync(~0u, sum, 2);
        // a lane's scores are of rows 2t and 2t + 1: what a product (in 2^-24) and the sum of
        // the query are multiplied by beside step and middle, and where a product starts.  (Step
        // and middle come times 2^11, which leaves these two below 2^127 scale: all in one of
        // them, queries above 2^117 gave infinity, whatever the keys.)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const float by = __shfl_sync(~0u, down, (2 * t + c) * 4) * mul0, all = __shfl_sync(~0u, sum, (2 * t + c) * 4);
            rowmul[n][c] = by * 0x1p13f, rowsum[n][c] = by * (all * 0x1p-11f), start[n][c] = -7.5f * 0x1p-24f * all;
            const int rw = row0 + 8 * n + 2 * t + c;
            const bool live_c = rw < rows;
            const int ii = live_c ? static_cast<int>(a.gdiv.div(rw)) : 0;
            prow[n][c] = q.p0 + ii;
            slope[n][c] = a.slopes && live_c ? a.slopes[h * a.G + rw - ii * a.G] * kLog2e : 0.0f;
            const RowMask m(a, q, prow[n][c], live_c);
            hi[n][c] = m.hi, from[n][c] = m.from, pre[n][c] = m.pre;
        }
    }

    if (NT > 1)
        __syncthreads();

    // outputs (in 2^-24; odd dimensions 16 times themselves plus the even one before); the sums of the rounded weights
    // in p (all four of its values), of weights over steps and of weights' middles
    float o[NT][MO][4], p_sum[NT][4];
    float m[NT][2], l[NT][2], mid[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int d = 0; d < MO; ++d)
            o[n][d][0] = o[n][d][1] = o[n][d][2] = o[n][d][3] = 0.0f;
        p_sum[n][0] = p_sum[n][1] = p_sum[n][2] = p_sum[n][3] = 0.0f;
        m[n][0] = m[n][1] = -INFINITY;
        l[n][0] = l[n][1] = mid[n][0] = mid[n][1] = 0.0f;
    }
    // where a lane's codes lie among a unit's: K's of key gid; V's row lane % 16, whose first 16
    // bytes are lanes 0 to 15's, the next the others' (16-byte pieces are swizzled by the row)
    const uint32_t k_at = D == 128 ? gid * 64 + ((t ^ (gid >> 1 & 3)) << 4) : gid * 32 + (((t >> 1) ^ (gid >> 2)) << 4 | (t & 1) << 3);
    const int v_turn = D == 128 ? lane >> 1 & 3 : lane >> 2 & 1;
    uint32_t v_at[D / 64];
#pragma unroll
    for (int g = 0; g < D / 64; ++g)
        v_at[g] = (lane & 15) * (D / 2) + (((2 * g + (lane >> 4)) ^ v_turn) << 4);
    const uint32_t ones[4] = {0x3c003c00u, 0x3c003c00u, 0x3c003c00u, 0x3c003c00u};

    unsigned batch = 0;
    for (unsigned it = 0; static_cast<int>(it) < n_it; ++it) {
        if (it / BI != batch) {
            batch = it / BI;
            cur = nxt;
            nxt = check(batch + 1, nid);
            nid = ask(batch + 2);
        }
        if (static_cast<int>(it) + ST - 1 < n_it)
            issue(it + ST - 1, batch);
        const int key = first_key(it);
        const unsigned units = units_of(cur, it);
        // (a lane that gives up takes its warp along: the others would meet it nowhere)
        if (!__all_sync(~0u, mbar_wait(bar0 + 8 * (it % ST), (it / ST) & 1, a.status))) {
            // give the loads in flight a while to land before the memory is used again
            for (unsigned k = it + 1; k < min(static_cast<unsigned>(n_it), it + ST); ++k)
                mbar_wait(bar0 + 8 * (k % ST), (k / ST) & 1, a.status, 2000000);
            __syncwarp();
            break;
        }
        if (units == 0)
            continue;                  // keys between the first ones and the window
        const uint32_t kt = ring + (it % ST) * S::stage, vt = kt + U * S::unit;
        const uint32_t *const num = reinterpret_cast<const uint32_t *>(base + (nums - sbase)) + it % ST * (2 * KW) + lane;

        // a lane a key: its numbers, and what its value's step gives its weights.  Those of
        // keys that a row does not see may be anything: their scores are replaced, and what
        // multiplies their weights of zero is finite (share_of always is).
#pragma unroll
        for (int x = 0; x < KW; x += 32) {
            const uint32_t kn = num[x], vn = num[KW + x];
            const float vs = value_scale(__uint_as_float(vn << 16)), share = share_of(vs);
            const float vmid = share * __uint_as_float(vn & 0xffff0000u);
            keys_s[x + lane] = make_float4(__uint_as_float(kn << 16) * 0x1p11f, __uint_as_float(kn & 0xffff0000u) * 0x1p11f, lg2(vs), share);
            mids_s[x + lane] = fabsf(vmid) <= 3.402823466e38f ? vmid : 0.0f;
        }

        // the units' keys gid and gid + 8; a unit that was not loaded gives
        // products of any codes, which no row sees
        float sc[U][NT][4];
#pragma unroll
        for (int u = 0; u < U; u += 2) {
            uint32_t kw[2][2][W];
#pragma unroll
            for (int v = 0; v < 2; ++v)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const uint32_t at = kt + (16 * (u + v) + 8 * x) * (D / 2) + k_at;
                    if (D == 128) {
                        const uint4 z = lds128(at);
                        kw[v][x][0] = z.x, kw[v][x][1] = z.y;
                        kw[v][x][W - 2] = z.z, kw[v][x][W - 1] = z.w;
                    } else {
                        const uint2 z = lds64(at);
                        kw[v][x][0] = z.x, kw[v][x][1] = z.y;
                    }
                }
#pragma unroll
            for (int w = 0; w < W; ++w) {
                uint32_t f[2][2][4];
#pragma unroll
                for (int v = 0; v < 2; ++v)
#pragma unroll
                    for (int x = 0; x < 2; ++x)
                        codes8_pairs(kw[v][x][w], f[v][x]);
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        uint2 qv;
                        if (NT > 1)
                            qv = q_s[(n * 2 * W + 2 * w + s) * 32 + lane];
                        else
                            qv = make_uint2(qf[2 * w + s][0], qf[2 * w + s][1]);
#pragma unroll
                        for (int v = 0; v < 2; ++v) {
                            const uint32_t g[4] = {f[v][0][2 * s], f[v][1][2 * s], f[v][0][2 * s + 1], f[v][1][2 * s + 1]};
                            if (w == 0 && s == 0)
                                mma16816_from(sc[u + v][n], g, qv.x, qv.y, start[n][0], start[n][1]);
                            else
                                mma16816(sc[u + v][n], g, qv.x, qv.y);
                        }
                    }
            }
        }

        // scores in base 2 with the logarithms of the values' steps
        __syncwarp();                  // keys_s
        const bool caps = a.softcap > 0.0f;
        float share[U][2], lvs[U][2];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const float4 num = keys_s[16 * u + gid + 8 * x];
                lvs[u][x] = num.z, share[u][x] = num.w;
                const float off = caps ? 0.0f : num.z;
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    float *const y = sc[u][n] + 2 * x;
                    float m0 = rowmul[n][0], m1 = rowmul[n][1], b0, b1;
                    mul2(m0, m1, num.x);
                    fma2(b0, b1, rowsum[n][0], rowsum[n][1], num.y, off);
                    fma2_each(y[0], y[1], y[0], y[1], m0, m1, b0, b1);
                }
            }
        auto each = [&](auto &&f) {
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        f(sc[u][n][e], n, e & 1, lvs[u][e >> 1], key + 16 * u + gid + 8 * (e >> 1));
        };
        if (caps) {
            if (plain_cap(a))
                each([&](float &y, int, int, float lv, int) {
                    y = fmaf(-2.0f * a.cap2, __fdividef(1.0f, 1.0f + ex2(y)), a.cap2 + lv);
                });
            else
                each([&](float &y, int, int, float lv, int) { y = capped(a, y) + lv; });
        }
        if (a.slopes)
            each([&](float &y, int n, int c, float, int j) { y = fmaf(slope[n][c], static_cast<float>(j - prow[n][c]), y); });
        // whether every row sees all of them (as all_see)
        if (!(key + KW <= first_end || (key + KW <= last_end && key >= begin)))
            each([&](float &y, int n, int c, float, int j) {
                y = (j < hi[n][c] && (j >= from[n][c] || j < a.sinks)) || j < pre[n][c] ? y : -INFINITY;
            });
        float mx[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n)
            mx[n][0] = mx[n][1] = -INFINITY;
        each([&](float &y, int n, int c, float, int) { mx[n][c] = fmaxf(mx[n][c], y); });
        // The reference moves, to the largest score so far, only when a weight would come out
        // above 2^15: mostly no maximum has to be joined over the lanes.
        bool up = false;
#pragma unroll
        for (int n = 0; n < NT; ++n)
            up |= mx[n][0] > m[n][0] + (15.0f - kPBits) || mx[n][1] > m[n][1] + (15.0f - kPBits);
        if (__any_sync(~0u, up)) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    float x = mx[n][c];
                    x = fmaxf(x, __shfl_xor_sync(~0u, x, 4));
                    x = fmaxf(x, __shfl_xor_sync(~0u, x, 8));
                    x = fmaxf(x, __shfl_xor_sync(~0u, x, 16));
                    const float mn = fmaxf(m[n][c], x), by = m[n][c] == mn ? 0.0f : m[n][c] - mn;
                    m[n][c] = mn;
                    // sums of weights over steps are scaled in two halves: counted up to 2^80 a
                    // weight (share_of), they outlast factors below float32's least
                    const float half = ex2(0.5f * by), f = half * half;
                    l[n][c] = l[n][c] * half * half, mid[n][c] = mid[n][c] * half * half;
                    p_sum[n][c] *= f, p_sum[n][2 + c] *= f;
#pragma unroll
                    for (int d = 0; d < MO; ++d)
                        o[n][d][c] *= f, o[n][d][2 + c] *= f;
                }
        }
        float mref[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int c = 0; c < 2; ++c)
                mref[n][c] = (m[n][c] == -INFINITY ? 0.0f : m[n][c]) - kPBits;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            // (a unit that was not loaded has weights of zero, and codes of any bytes)
            uint32_t pf[NT][2];
            const float vmid[2] = {mids_s[16 * u + gid], mids_s[16 * u + gid + 8]};
#pragma unroll
            for (int n = 0; n < NT; ++n) {
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    float p[2] = {sc[u][n][2 * x], sc[u][n][2 * x + 1]};
                    add2(p[0], p[1], -mref[n][0], -mref[n][1]);
                    p[0] = ex2(p[0]), p[1] = ex2(p[1]);
                    acc2(l[n][0], l[n][1], p[0], p[1], share[u][x]);
                    acc2(mid[n][0], mid[n][1], p[0], p[1], vmid[x]);
                    pf[n][x] = transpose8(pack_half(p[0], p[1]));
                }
                mma16816(p_sum[n], ones, pf[n][0], pf[n][1]);
            }
            // Value rows 2t and 2t + 1, and 2t + 8 and 2t + 9, of the unit: four codes of either as
            // one 16-bit element each, dimensions 4 gid to 4 gid + 3 of every 32.
#pragma unroll
            for (int g = 0; g < D / 64; ++g) {
                uint32_t x[4];
                ldmatrix4_trans(x, vt + u * S::unit + v_at[g]);
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    // rows gid and gid + 8 of two tiles: a dimension and the next, and the two behind
                    uint32_t f0[4], f1[4];
                    codes4_pairs(x[2 * e], f0);
                    codes4_pairs(x[2 * e + 1], f1);
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const uint32_t f[4] = {f0[2 * y], f0[2 * y + 1], f1[2 * y], f1[2 * y + 1]};
#pragma unroll
                        for (int n = 0; n < NT; ++n)
                            mma16816(o[n][4 * g + 2 * e + y], f, pf[n][0], pf[n][1]);
                    }
                }
            }
        }
        __syncwarp();                  // the stage is free: the next issue may overwrite it
    }

    // outputs in units of one, with the middles
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            float x = mid[n][c];
            x += __shfl_xor_sync(~0u, x, 4);
            x += __shfl_xor_sync(~0u, x, 8);
            x += __shfl_xor_sync(~0u, x, 16);
            // (middles count as weights do, by kRef)
            const float add = fmaf(-7.5f, p_sum[n][c], x * (1.0f / kRef));
#pragma unroll
            for (int d = 0; d < MO; ++d) {
                o[n][d][2 + c] = fmaf(o[n][d][2 + c] - o[n][d][c], 0x1p20f, add);
                o[n][d][c] = fmaf(o[n][d][c], 0x1p24f, add);
            }
        }
    finish_rows<D, T, NT, true>(a, q, base, ml, m, l, o, h, split, row0, rows, bad);
}

template <int D, typename T, int NT>
cudaError_t step4_rows(const fkv_ctx *ctx, const AttendArgs &a, const CUtensorMap &mk, const CUtensorMap &mv, cudaStream_t st)
{
    constexpr int smem = Step4Shape<D, NT>::smem;
    // the block's end takes the rings' place: the warps' outputs, and a cluster's shares
    static_assert(4 * 8 * NT * (D + 4) * 4 + 8 * NT * (D + 1) * 4 <= Step4Shape<D, NT>::ring, "the ring holds the outputs");
    const void *fn = reinterpret_cast<const void *>(k_attend_step4<D, T, NT>);
    const cudaError_t e = kernel_use(ctx, fn, 128, smem, nullptr);
    if (e != cudaSuccess)
        return e;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = a.cluster ? a.splits : 1, at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(a.n_req * a.row_tiles * a.splits), a.H), cfg.blockDim = dim3(128);
    cfg.dynamicSmemBytes = smem, cfg.stream = st;
    cfg.attrs = &at, cfg.numAttrs = a.cluster ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, k_attend_step4<D, T, NT>, a, mk, mv);
}

template <int D, typename T>
cudaError_t step4_nt(const fkv_ctx *ctx, const AttendArgs &a, int nt, const CUtensorMap &mk, const CUtensorMap &mv, cudaStream_t st)
{
    return nt == 1 ? step4_rows<D, T, 1>(ctx, a, mk, mv, st) : step4_rows<D, T, 2>(ctx, a, mk, mv, st);
}

}  // namespace

cudaError_t launch_attend_step4(const fkv_ctx *ctx, const AttendArgs &a, int dim, int dtype, int nt, const CUtensorMap &mk,
                                const CUtensorMap &mv, cudaStream_t st)
{
    if (dim == 64)
        return dtype == FKV_F16 ? step4_nt<64, __half>(ctx, a, nt, mk, mv, st) : step4_nt<64, __nv_bfloat16>(ctx, a, nt, mk, mv, st);
    return dtype == FKV_F16 ? step4_nt<128, __half>(ctx, a, nt, mk, mv, st) : step4_nt<128, __nv_bfloat16>(ctx, a, nt, mk, mv, st);
}
