// Attention over the paged 8-bit K/V cache (fkv_page_attend).
//
// For a query row (token i of request r, query head u of KV head h) at position
// p = kv_len - n_new + i, with c the codes of a page and ks, vs its scales,
//     x_j = f(scale ks q.c_j) + slope (j - p),   f(s) = cap tanh(s / cap) or s
//     o   = sum_j exp(x_j) vs c'_j / sum_j exp(x_j)   over the visible j.
// Codes are exact in fp16, and so is a query row brought to [2^14, 2^15) by a
// power of two (fp16 queries as they are): the products are exact and summed in
// fp32 on the tensor cores, and the scale of a page multiplies afterwards, once
// for each score.  The value scale goes into the softmax instead: with
//     y_j = x_j log2 e + log2 vs,    P_j = 2^(y_j - m + 8),   m = max y_j
// the second product is sum P_j c'_j with P rounded to fp16 (relative 2^-11, an
// eighth of a bf16 result's own rounding; P spans 2^8 .. 2^-24, so nothing above
// 2^-32 of the largest weight is lost), and the sum of the weights is
// sum P_j / vs, from the unrounded P_j, in fp32.  So pages of any scales mix in
// one accumulator without a rounding of V.
#include <type_traits>

#include "paged.cuh"

using namespace fkvd;

namespace {

constexpr int kTile = 128;         // keys a tile: the unit of the visible range and of the splits
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kPBits = 8.0f;     // P is at most 2^8

struct AttendArgs {
    const void *q;
    void *out;
    float *lse;
    const int *cu, *kv_len, *table;
    const float *ks, *vs, *slopes;
    const int *prefix;
    float *ws_o, *ws_lse;
    unsigned *status;
    int64_t q_tok, q_head, o_tok, o_head, table_stride, scb, sch, n_blocks, T;
    int n_req, H, G, block, width, max_new, max_len, window, sinks, causal;
    int splits, chunk, row_tiles;
    float scale, softcap;
    FastDiv div, gdiv;
};

// What one request's rows see.
struct Request {
    int tok0, nq, len, pre, p0;
    // false: the request's numbers do not hold together; it is reported and skipped
    __device__ __forceinline__ bool load(const AttendArgs &a, int r)
    {
        const int c0 = a.cu[r], c1 = a.cu[r + 1];
        len = a.kv_len[r];
        tok0 = c0;
        nq = c1 - c0;
        pre = a.prefix ? min(max(a.prefix[r], 0), len) : 0;
        p0 = len - nq;
        return c0 >= 0 && c1 >= c0 && c1 <= a.T && nq <= a.max_new && len >= 0 && len <= a.max_len &&
               static_cast<int64_t>(len) <= static_cast<int64_t>(a.width) * a.block;
    }
};

// The tiles that rows at positions pa .. pb see: those of the first `lo`
// positions (prefix, sinks), then those from the window's beginning on.
struct Tiles {
    int n_lo, hi0, n, lim;
    __device__ __forceinline__ Tiles(const AttendArgs &a, const Request &q, int pa, int pb)
    {
        const int end = pb < 0 ? 0 : (a.causal ? min(q.len, pb + 1) : q.len);
        const int lo = pb < 0 ? 0 : max(q.pre, a.window ? min(a.sinks, end) : 0);
        const int begin = a.window ? max(0, pa - a.window + 1) : 0;
        lim = max(end, lo);
        n_lo = (lo + kTile - 1) / kTile;
        hi0 = max(n_lo, begin / kTile);
        n = n_lo + max(0, (end + kTile - 1) / kTile - hi0);
    }
    __device__ __forceinline__ int at(int i) const { return i < n_lo ? i : hi0 + i - n_lo; }
};

// The keys that one row sees: j < hi and (j >= from or j < sinks), or j < pre.
struct RowMask {
    int hi, from, pre;
    __device__ __forceinline__ RowMask(const AttendArgs &a, const Request &q, int p, bool live)
    {
        const bool on = live && p >= 0;
        hi = on ? (a.causal ? min(q.len, p + 1) : q.len) : 0;
        from = a.window ? p - a.window + 1 : 0;
        pre = on ? q.pre : 0;
    }
    __device__ __forceinline__ bool sees(const AttendArgs &a, int j) const
    {
        return (j < hi && (j >= from || j < a.sinks)) || j < pre;
    }
};

// Whether every row at positions pa .. pb sees all of [k0, k1).
__device__ __forceinline__ bool all_see(const AttendArgs &a, const Request &q, int pa, int pb, int k0, int k1)
{
    return pa >= 0 && k1 <= q.len &&
           (k1 <= q.pre || ((!a.causal || k1 - 1 <= pa) && (!a.window || k0 > pb - a.window || k1 <= a.sinks)));
}

__device__ __forceinline__ float cap_tanh(float s, float cap)
{
    // tanh x = 1 - 2 / (1 + e^2x): an absolute error of a few 2^-24
    return cap * (1.0f - __fdividef(2.0f, 1.0f + ex2(s * (2.0f * kLog2e) / cap)));
}

__device__ __forceinline__ void mma16816(float *c, const uint32_t *a, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap *map, int c0, int c1, int c2, int c3,
                                            uint32_t bar)
{
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(bar)
        : "memory");
}

__device__ __forceinline__ uint4 lds128(uint32_t a)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
    return v;
}

__device__ __forceinline__ uint2 lds64(uint32_t a)
{
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a));
    return v;
}

__device__ __forceinline__ uint32_t pack_half(float a, float b)
{
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}

// Finished (or partial) row: o, lse to the outputs or to the workspace.
template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// ------------------------------------------------------------------ steps --
// Up to 16 rows (the query heads of a KV head, times the new tokens) against a
// share of the keys: bound by reading the pages.  A warp owns every fourth
// group of 32 keys, loads it by TMA into a ring of its own and keeps its own
// running maximum, sum and output, so nothing but the last merge joins the
// warps.  Codes go from shared memory to the tensor cores' fragments through
// registers (the contraction may run over the head dimension in any order, so a
// lane takes 16 consecutive bytes of a key as four steps' operands; a value
// row's 16 bytes are 16 columns of the result).  mma.sync, as 16 rows are an
// eighth of what tcgen05 multiplies at least: its rate is four times what the
// bytes leave time for.
template <int D> struct StepShape {
    static constexpr int stages = D == 128 ? 3 : 6;
    static constexpr int smem = 4 * stages * 64 * D + 1024;
};

template <int D, int FMT, typename T>
__global__ void __launch_bounds__(128, 2)
    k_attend_step(const AttendArgs a, const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv)
{
    constexpr int ST = StepShape<D>::stages, NS = D / 64, UNIT = 16 * D, STAGE = 4 * UNIT, NO = D / 8;
    extern __shared__ uint8_t raw[];
    __shared__ __align__(8) uint64_t bars[4 * ST];
    __shared__ float ml[4][2][16];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, gid = lane >> 2, t = lane & 3;
    const uint32_t sbase = (smem_u32(raw) + 1023) & ~1023u;

    const int h = blockIdx.y;
    const int split = blockIdx.x % a.splits, rr = blockIdx.x / a.splits;
    const int rt = rr % a.row_tiles, r = rr / a.row_tiles;
    Request q;
    if (!q.load(a, r)) {
        if (tid == 0)
            atomicOr(a.status, FKV_ST_RANGE);
        return;
    }
    const int rows = q.nq * a.G, row0 = rt * 16;
    if (row0 >= rows)
        return;
    const int ia = static_cast<int>(a.gdiv.div(row0)), ib = static_cast<int>(a.gdiv.div(min(row0 + 15, rows - 1)));
    const int pa = q.p0 + ia, pb = q.p0 + ib;
    const Tiles tiles(a, q, pa, pb);
    const int i0 = split * a.chunk, i1 = min(tiles.n, i0 + a.chunk);

    const uint32_t ring = sbase + warp * ST * STAGE, bar0 = smem_u32(bars) + warp * ST * 8;
    if (lane == 0) {
        for (int s = 0; s < ST; ++s)
            mbar_init(bar0 + 8 * s, 1);
        fence_mbar_init();
    }
    __syncwarp();

    // page ids and scales of the next 16 iterations' units, two a lane pair
    int id_c = -1, id_n = -1;
    float ks_c = 0.0f, vs_c = 1.0f, ks_n = 0.0f, vs_n = 1.0f;
    bool bad = false;
    auto fetch = [&](int batch, int &id, float &ks, float &vs) {
        const int it = i0 + batch * 16 + (lane >> 1);
        id = -1, ks = 0.0f, vs = 1.0f;
        if (it < i1) {
            const int key = tiles.at(it) * kTile + warp * 32 + (lane & 1) * 16;
            if (key < tiles.lim) {
                id = a.table[r * a.table_stride + a.div.div(key)];
                if (id < 0 || id >= a.n_blocks) {
                    bad = true;
                    id = 0;
                }
                ks = a.ks[id * a.scb + h * a.sch];
                vs = a.vs[id * a.scb + h * a.sch];
            }
        }
    };
    const int n_it = max(0, i1 - i0);
    fetch(0, id_c, ks_c, vs_c);
    fetch(1, id_n, ks_n, vs_n);
    // units of iteration `it` that hold keys to look at
    auto units = [&](int it) {
        const int key = tiles.at(i0 + it) * kTile + warp * 32;
        return key >= tiles.lim ? 0 : (key + 16 >= tiles.lim ? 1 : 2);
    };
    auto issue = [&](int it, int batch) {
        const int nu = units(it);
        const int from = (it & 15) * 2;
        const int ids[2] = {__shfl_sync(~0u, (it >> 4) == batch ? id_c : id_n, from),
                            __shfl_sync(~0u, (it >> 4) == batch ? id_c : id_n, from + 1)};
        if (lane == 0 && nu) {
            const uint32_t bar = bar0 + 8 * (it % ST), dst = ring + (it % ST) * STAGE;
            mbar_arrive_expect_tx(bar, nu * 2 * UNIT);
            const int key = tiles.at(i0 + it) * kTile + warp * 32;
            for (int u = 0; u < nu; ++u) {
                const int k0 = key + 16 * u, off = k0 - static_cast<int>(a.div.div(k0)) * a.block;
                tma_load_4d(dst + u * UNIT, &mk, 0, off, h, ids[u], bar);
                tma_load_4d(dst + (2 + u) * UNIT, &mv, 0, off, h, ids[u], bar);
            }
        }
        __syncwarp();
    };
    for (int it = 0; it < min(ST - 1, n_it); ++it)
        issue(it, 0);

    // the query rows as fp16 fragments: lane t's steps take 16 consecutive
    // dimensions (two such pieces for D = 128) of rows gid and gid + 8
    uint32_t qf[NS * 4][4];
    float rowmul[2], slope[2];
    int prow[2];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const int row = row0 + gid + 8 * half;
        const bool live = row < rows;
        const int i = live ? static_cast<int>(a.gdiv.div(row)) : 0, u = live ? row - i * a.G : 0;
        const T *src = static_cast<const T *>(a.q) + (q.tok0 + i) * a.q_tok + (h * a.G + u) * a.q_head;
        float x[NS][16];
        float amax = 0.0f;
#pragma unroll
        for (int s = 0; s < NS; ++s) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                uint4 v = make_uint4(0, 0, 0, 0);
                if (live)
                    v = *reinterpret_cast<const uint4 *>(src + (NS * t + s) * 16 + 8 * e);
                const T *y = reinterpret_cast<const T *>(&v);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    x[s][8 * e + k] = static_cast<float>(y[k]);
                    amax = fmaxf(amax, fabsf(x[s][8 * e + k]));
                }
            }
        }
        amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, 1));
        amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, 2));
        // bf16 rows: 2^(14 - exponent), so that fp16 holds them (see above)
        float up = 1.0f, down = 1.0f;
        if (sizeof(T) == 2 && !(std::is_same<T, __half>::value) && amax > 0.0f) {
            const int e = max(static_cast<int>(__float_as_uint(amax) >> 23) - 127, -100);
            up = __uint_as_float(static_cast<uint32_t>(127 + 14 - e) << 23);
            down = __uint_as_float(static_cast<uint32_t>(127 - 14 + e) << 23);
        }
        rowmul[half] = a.scale * down;
        prow[half] = q.p0 + i;
        slope[half] = a.slopes && live ? a.slopes[h * a.G + u] * kLog2e : 0.0f;
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
                qf[s * 4 + kk][half] = pack_half(x[s][4 * kk] * up, x[s][4 * kk + 1] * up);
                qf[s * 4 + kk][2 + half] = pack_half(x[s][4 * kk + 2] * up, x[s][4 * kk + 3] * up);
            }
    }
    const RowMask mask0(a, q, prow[0], row0 + gid < rows), mask1(a, q, prow[1], row0 + gid + 8 < rows);

    float o[NO][4];
#pragma unroll
    for (int n = 0; n < NO; ++n)
        o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.0f;
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f};

    int batch = 0;
    for (int it = 0; it < n_it; ++it) {
        if ((it >> 4) != batch) {
            batch = it >> 4;
            id_c = id_n, ks_c = ks_n, vs_c = vs_n;
            fetch(batch + 1, id_n, ks_n, vs_n);
        }
        if (it + ST - 1 < n_it)
            issue(it + ST - 1, batch);
        const int nu = units(it);
        if (!nu)
            break;                      // the last tile's end
        if (!mbar_wait(bar0 + 8 * (it % ST), (it / ST) & 1, a.status))
            break;
        const uint32_t kt = ring + (it % ST) * STAGE, vt = kt + 2 * UNIT;
        const int key = tiles.at(i0 + it) * kTile + warp * 32;

        float sc[4][4];
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            sc[n][0] = sc[n][1] = sc[n][2] = sc[n][3] = 0.0f;
            if ((n >> 1) < nu) {
                const int kr = 8 * n + gid;
#pragma unroll
                for (int s = 0; s < NS; ++s) {
                    const int c = NS * t + s;
                    const uint32_t at = D == 128 ? kr * 128 + ((c ^ (kr & 7)) << 4) : kr * 64 + ((c ^ ((kr >> 1) & 3)) << 4);
                    const uint4 w = lds128(kt + at);
                    const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk) {
                        uint32_t b0, b1;
                        codes4_half<FMT>(ww[kk], b0, b1);
                        mma16816(sc[n], qf[s * 4 + kk], b0, b1);
                    }
                }
            }
        }

        // scores, masks and the value scales' logarithms
        const bool full = all_see(a, q, pa, pb, key, key + 16 * nu);
        float mx[2] = {-INFINITY, -INFINITY}, ivs[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const float ks = __shfl_sync(~0u, ks_c, (it & 15) * 2 + u);
            const float vs = fmaxf(__shfl_sync(~0u, vs_c, (it & 15) * 2 + u), FKV_PAGE_MIN_SCALE);
            const float lvs = lg2(vs);
            ivs[u] = __frcp_rn(vs);
#pragma unroll
            for (int n = 2 * u; n < 2 * u + 2; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int half = e >> 1, j = key + 8 * n + 2 * t + (e & 1);
                    float x = sc[n][e] * (ks * rowmul[half]);
                    if (a.softcap > 0.0f)
                        x = cap_tanh(x, a.softcap);
                    x = x * kLog2e;
                    if (a.slopes)
                        x += slope[half] * static_cast<float>(j - prow[half]);
                    x += lvs;
                    if (u >= nu || (!full && !(half ? mask1 : mask0).sees(a, j)))
                        x = -INFINITY;
                    sc[n][e] = x;
                    mx[half] = fmaxf(mx[half], x);
                }
        }
        float alpha[2], mref[2];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            mx[half] = fmaxf(mx[half], __shfl_xor_sync(~0u, mx[half], 1));
            mx[half] = fmaxf(mx[half], __shfl_xor_sync(~0u, mx[half], 2));
            const float mn = fmaxf(m[half], mx[half]);
            mref[half] = mn == -INFINITY ? 0.0f : mn;
            alpha[half] = ex2(m[half] - mref[half]);
            m[half] = mn;
            l[half] *= alpha[half];
        }
        if (__any_sync(~0u, alpha[0] != 1.0f || alpha[1] != 1.0f)) {
#pragma unroll
            for (int n = 0; n < NO; ++n) {
                o[n][0] *= alpha[0], o[n][1] *= alpha[0];
                o[n][2] *= alpha[1], o[n][3] *= alpha[1];
            }
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            if (u >= nu)
                break;
            uint32_t pf[4];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int n = 2 * u + x;
                float p[4];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    p[e] = ex2(sc[n][e] - mref[e >> 1] + kPBits);
                l[0] += (p[0] + p[1]) * ivs[u];
                l[1] += (p[2] + p[3]) * ivs[u];
                pf[2 * x] = pack_half(p[0], p[1]);
                pf[2 * x + 1] = pack_half(p[2], p[3]);
            }
            // value rows 2t, 2t + 1, 2t + 8, 2t + 9 of the unit; those behind the
            // request's end hold any bytes, NaN codes among them: read as zeros
            const int vr[4] = {2 * t, 2 * t + 1, 2 * t + 8, 2 * t + 9};
            const bool tail = key + 16 * u + 16 > q.len;
            uint32_t w[4][D / 32];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int row = 16 * u + vr[x];
                if (D == 128) {
                    const uint4 v = lds128(vt + row * 128 + ((gid ^ (row & 7)) << 4));
                    w[x][0] = v.x, w[x][1] = v.y;
                    if (D == 128)
                        w[x][D / 32 - 2] = v.z, w[x][D / 32 - 1] = v.w;
                } else {
                    const uint2 v = lds64(vt + row * 64 + ((((gid >> 1) ^ ((row >> 1) & 3)) << 4) | (gid & 1) << 3));
                    w[x][0] = v.x, w[x][1] = v.y;
                }
                if (tail && key + row >= q.len) {
#pragma unroll
                    for (int k = 0; k < D / 32; ++k)
                        w[x][k] = 0;
                }
            }
#pragma unroll
            for (int k = 0; k < D / 32; ++k) {
                uint32_t b0[4], b1[4];
                codes4_half<FMT>(__byte_perm(w[0][k], w[1][k], 0x5140), b0[0], b0[1]);
                codes4_half<FMT>(__byte_perm(w[0][k], w[1][k], 0x7362), b0[2], b0[3]);
                codes4_half<FMT>(__byte_perm(w[2][k], w[3][k], 0x5140), b1[0], b1[1]);
                codes4_half<FMT>(__byte_perm(w[2][k], w[3][k], 0x7362), b1[2], b1[3]);
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    mma16816(o[4 * k + c], pf, b0[c], b1[c]);
            }
        }
        __syncwarp();                  // the stage is free: the next issue may overwrite it
    }

    // merge the warps: a row's largest m, then sums and outputs against it
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        l[half] += __shfl_xor_sync(~0u, l[half], 1);
        l[half] += __shfl_xor_sync(~0u, l[half], 2);
        if (t == 0) {
            ml[warp][0][gid + 8 * half] = m[half];
            ml[warp][1][gid + 8 * half] = l[half];
        }
    }
    __syncthreads();                   // every ring is read: its memory takes the outputs
    float *mo = reinterpret_cast<float *>(raw + (sbase - smem_u32(raw)));
    constexpr int LD = D + 4;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        float *dst = mo + (warp * 16 + gid + 8 * half) * LD;
        // n-tile n, column c of the fragments is dimension c * (D / 8) + n
#pragma unroll
        for (int n = 0; n < NO; ++n) {
            dst[2 * t * NO + n] = o[n][2 * half];
            dst[(2 * t + 1) * NO + n] = o[n][2 * half + 1];
        }
    }
    __syncthreads();
    if (bad)
        atomicOr(a.status, FKV_ST_RANGE);
    // thread: row tid / 8, dimensions (tid % 8) * D / 8 on
    {
        const int row = tid >> 3, c = (tid & 7) * (D / 8);
        if (row0 + row < rows) {
            float mt = -INFINITY;
#pragma unroll
            for (int w = 0; w < 4; ++w)
                mt = fmaxf(mt, ml[w][0][row]);
            const float mref = mt == -INFINITY ? 0.0f : mt;
            float lt = 0.0f, f[4];
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                f[w] = ex2(ml[w][0][row] - mref);
                lt += ml[w][1][row] * f[w];
            }
            const float inv = lt > 0.0f ? 1.0f / lt : 0.0f;
            const float lse2 = lt > 0.0f ? mref - kPBits + log2f(lt) : -INFINITY;
            const int i = static_cast<int>(a.gdiv.div(row0 + row)), u = row0 + row - i * a.G;
            const int64_t tok = q.tok0 + i, head = h * a.G + u, flat = tok * (a.H * a.G) + head;
            float x[D / 8];
#pragma unroll
            for (int k = 0; k < D / 8; ++k) {
                x[k] = 0.0f;
#pragma unroll
                for (int w = 0; w < 4; ++w)
                    x[k] += mo[(w * 16 + row) * LD + c + k] * f[w];
                x[k] *= inv;
            }
            if (a.splits == 1) {
                T *dst = static_cast<T *>(a.out) + tok * a.o_tok + head * a.o_head + c;
                T y[D / 8];
#pragma unroll
                for (int k = 0; k < D / 8; ++k)
                    y[k] = from_float<T>(x[k]);
#pragma unroll
                for (int k = 0; k < D / 64; ++k)
                    reinterpret_cast<uint4 *>(dst)[k] = reinterpret_cast<const uint4 *>(y)[k];
                if (a.lse && c == 0)
                    a.lse[flat] = lse2 / kLog2e;
            } else {
                const int64_t at = split * a.T * (a.H * a.G) + flat;
                float *dst = a.ws_o + at * D + c;
#pragma unroll
                for (int k = 0; k < D / 32; ++k)
                    reinterpret_cast<float4 *>(dst)[k] = make_float4(x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]);
                if (c == 0)
                    a.ws_lse[at] = lse2;
            }
        }
    }
}

// --------------------------------------------------------------- combine --
// A warp per query row: the splits' outputs weighted by 2^(lse - largest).
template <int D, typename T> __global__ void __launch_bounds__(128) k_attend_combine(const AttendArgs a)
{
    const int lane = threadIdx.x & 31;
    const int64_t Hq = a.H * a.G, row = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 5);
    // rows behind the last request's are no one's, and rows of a request that
    // was skipped have no partial results: both are left as they are
    if (row >= a.T * Hq)
        return;
    const int64_t tok = row / Hq, head = row - tok * Hq;
    int lo = 0, hi = a.n_req;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.cu[mid] <= tok)
            lo = mid;
        else
            hi = mid;
    }
    Request q;
    if (!q.load(a, lo) || tok < q.tok0 || tok >= q.tok0 + q.nq)
        return;
    float mx = -INFINITY;
    for (int s = lane; s < a.splits; s += 32)
        mx = fmaxf(mx, a.ws_lse[s * a.T * Hq + row]);
#pragma unroll
    for (int o = 16; o; o >>= 1)
        mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, o));
    const float mref = mx == -INFINITY ? 0.0f : mx;
    constexpr int E = D / 32;
    float x[E], sum = 0.0f;
#pragma unroll
    for (int k = 0; k < E; ++k)
        x[k] = 0.0f;
    for (int s = 0; s < a.splits; ++s) {
        const int64_t at = s * a.T * Hq + row;
        const float w = ex2(a.ws_lse[at] - mref);
        if (w == 0.0f)
            continue;
        sum += w;
#pragma unroll
        for (int k = 0; k < E; ++k)
            x[k] += w * a.ws_o[at * D + lane * E + k];
    }
    const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
    T *dst = static_cast<T *>(a.out) + tok * a.o_tok + head * a.o_head + lane * E;
#pragma unroll
    for (int k = 0; k < E; ++k)
        dst[k] = from_float<T>(x[k] * inv);
    if (a.lse && lane == 0)
        a.lse[row] = sum > 0.0f ? (mref + log2f(sum)) / kLog2e : -INFINITY;
}

// ------------------------------------------------------------------ launch --
struct Plan {
    int row_tiles, splits, chunk;
};

// How many shares the keys are split into.  A block's time is its keys plus a
// fixed part (its launch, the first loads' latency and the merge: about that
// of 384 keys); the blocks run in waves of `slots`.  The split with the least
// waves x time wins; joining the partial results costs another part a split.
Plan plan_of(const fkv_ctx *ctx, int64_t n_req, int H, int G, int64_t max_new, int64_t max_len, int window)
{
    Plan p;
    p.row_tiles = static_cast<int>((max_new * G + 15) / 16);
    const int64_t blocks = n_req * H * p.row_tiles, slots = ctx->sms * 2;
    int64_t span = max_len;
    if (window && window + max_new + 2 * kTile < span)
        span = window + max_new + 2 * kTile;
    const int tiles = static_cast<int>((span + kTile - 1) / kTile);
    double best = 0.0;
    p.splits = 1;
    p.chunk = tiles > 0 ? tiles : 1;
    for (int s = 1; s <= 64 && s <= tiles; ++s) {
        const int chunk = (tiles + s - 1) / s;
        const int64_t waves = (blocks * s + slots - 1) / slots;
        const double cost = waves * (chunk * kTile + 384.0) + (s > 1 ? 512.0 + 8.0 * s : 0.0);
        if (s == 1 || cost < best) {
            best = cost;
            p.splits = (tiles + chunk - 1) / chunk;
            p.chunk = chunk;
        }
    }
    return p;
}

// A window that holds every position is none.
int window_of(const fkv_attend *opt)
{
    return opt->window >= FKV_PAGE_MAX_LEN ? 0 : static_cast<int>(opt->window);
}

template <int D, int FMT, typename T>
cudaError_t step_as(const fkv_ctx *ctx, const AttendArgs &a, const CUtensorMap &mk, const CUtensorMap &mv, cudaStream_t st)
{
    const void *fn = reinterpret_cast<const void *>(k_attend_step<D, FMT, T>);
    cudaError_t e = kernel_use(ctx, fn, 128, StepShape<D>::smem, nullptr);
    if (e != cudaSuccess)
        return e;
    const dim3 grid(static_cast<unsigned>(a.n_req * a.row_tiles * a.splits), a.H);
    k_attend_step<D, FMT, T><<<grid, 128, StepShape<D>::smem, st>>>(a, mk, mv);
    e = cudaGetLastError();
    if (e != cudaSuccess || a.splits == 1)
        return e;
    k_attend_combine<D, T><<<static_cast<unsigned>((a.T * a.H * a.G + 3) / 4), 128, 0, st>>>(a);
    return cudaGetLastError();
}

template <int D, int FMT>
cudaError_t step_dt(const fkv_ctx *ctx, const AttendArgs &a, int dtype, const CUtensorMap &mk, const CUtensorMap &mv,
                    cudaStream_t st)
{
    return dtype == FKV_F16 ? step_as<D, FMT, __half>(ctx, a, mk, mv, st)
                            : step_as<D, FMT, __nv_bfloat16>(ctx, a, mk, mv, st);
}

}  // namespace

int64_t page_attend_workspace(const fkv_ctx *ctx, const fkv_pages *pg, int64_t n_req, int n_q_heads, int64_t T,
                              int64_t max_new, int64_t max_len, const fkv_attend *opt)
{
    const Plan p = plan_of(ctx, n_req, pg->n_heads, n_q_heads / pg->n_heads, max_new, max_len, window_of(opt));
    if (p.splits == 1)
        return 0;
    return (static_cast<int64_t>(p.splits) * T * n_q_heads * (pg->dim + 1) * 4 + 255) / 256 * 256;
}

cudaError_t launch_page_attend(const fkv_ctx *ctx, const fkv_pages *pg, const fkv_rows *q, int64_t T, int n_q_heads,
                               const int32_t *cu, const int32_t *kv_len, int64_t n_req, const int32_t *table,
                               int64_t table_stride, int64_t width, int64_t max_new, int64_t max_len,
                               const fkv_attend *opt, const fkv_rows *out, float *lse, void *ws,
                               const CUtensorMap &mk, const CUtensorMap &mv, cudaStream_t st)
{
    AttendArgs a;
    a.q = q->data, a.out = out->data, a.lse = lse;
    a.cu = cu, a.kv_len = kv_len, a.table = table;
    a.ks = pg->k_scale, a.vs = pg->v_scale, a.slopes = opt->slopes, a.prefix = opt->prefix;
    a.status = ctx->d_status;
    a.q_tok = q->stride_tok, a.q_head = q->stride_head, a.o_tok = out->stride_tok, a.o_head = out->stride_head;
    a.table_stride = table_stride, a.scb = pg->scale_stride_block, a.sch = pg->scale_stride_head;
    a.n_blocks = pg->n_blocks, a.T = T;
    a.n_req = static_cast<int>(n_req), a.H = pg->n_heads, a.G = n_q_heads / pg->n_heads, a.block = pg->block;
    a.width = static_cast<int>(width), a.max_new = static_cast<int>(max_new), a.max_len = static_cast<int>(max_len);
    a.window = window_of(opt);
    a.sinks = a.window ? static_cast<int>(opt->sinks < FKV_PAGE_MAX_LEN ? opt->sinks : FKV_PAGE_MAX_LEN) : 0;
    a.causal = opt->causal;
    a.scale = opt->scale, a.softcap = opt->softcap;
    a.div = FastDiv::make(pg->block), a.gdiv = FastDiv::make(a.G);
    const Plan p = plan_of(ctx, n_req, a.H, a.G, max_new, max_len, a.window);
    a.row_tiles = p.row_tiles, a.splits = p.splits, a.chunk = p.chunk;
    a.ws_o = static_cast<float *>(ws);
    a.ws_lse = a.ws_o ? a.ws_o + static_cast<int64_t>(p.splits) * T * n_q_heads * pg->dim : nullptr;
    const bool i8 = pg->format == FKV_INT8;
    if (pg->dim == 64)
        return i8 ? step_dt<64, FKV_INT8>(ctx, a, q->dtype, mk, mv, st) : step_dt<64, FKV_E4M3>(ctx, a, q->dtype, mk, mv, st);
    return i8 ? step_dt<128, FKV_INT8>(ctx, a, q->dtype, mk, mv, st) : step_dt<128, FKV_E4M3>(ctx, a, q->dtype, mk, mv, st);
}
