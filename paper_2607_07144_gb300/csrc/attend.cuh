// What the two attention kernels over the paged cache share (attend.cu,
// attend_prompt.cu): arguments, the visible range of a request's rows, and how
// the value scales enter.
#pragma once

#include <type_traits>

#include "paged.cuh"

namespace fkvd {

constexpr int kTile = 128;         // keys a tile: the unit of the visible range and of the splits
constexpr float kLog2e = 1.4426950408889634f;

struct AttendArgs {
    const void *q, *pool_k, *pool_v;
    void *out;
    float *lse;
    const int *cu, *kv_len, *table;
    const float *ks, *vs, *slopes;
    const int *prefix;
    float *ws_o, *ws_lse;
    unsigned *status;
    int64_t q_tok, q_head, o_tok, o_head, table_stride, sb, sh, st, scb, sch, n_blocks, T;
    int n_req, H, G, block, width, max_new, max_len, window, sinks, causal;
    int splits, chunk, row_tiles;
    bool cluster;                // a row's splits are one cluster, which joins them
    float scale, softcap;
    float cap2, cap_inv;         // cap log2 e and its reciprocal
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

// What some rows see: the first `lo` positions (prefix, sinks), and those from
// `begin` to `end` (the window's).
struct Seen {
    int lo, begin, end;
    // Whether any of the rows sees one of the 16 keys from k on.  Others of a tile are
    // not looked up: their pages may be gone.
    __device__ __forceinline__ bool of(int k) const { return k < lo || (k + 16 > begin && k < end); }
};

// The tiles that rows at positions pa .. pb see: the first positions', then the window's.
struct Tiles {
    Seen seen;
    int n_lo, hi0, n, lim;
    __device__ __forceinline__ Tiles(const AttendArgs &a, const Request &q, int pa, int pb)
    {
        const int end = pb < 0 ? 0 : (a.causal ? min(q.len, pb + 1) : q.len);
        const int lo = pb < 0 ? 0 : max(q.pre, a.window ? min(a.sinks, end) : 0);
        const int begin = a.window ? max(0, pa - a.window + 1) : 0;
        seen = {lo, begin, end};
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
};

// Whether every row at positions pa .. pb sees all of [k0, k1).
__device__ __forceinline__ bool all_see(const AttendArgs &a, const Request &q, int pa, int pb, int k0, int k1)
{
    return pa >= 0 && k1 <= q.len &&
           (k1 <= q.pre || ((!a.causal || k1 - 1 <= pa) && (!a.window || k0 > pb - a.window || k1 <= a.sinks)));
}

__device__ __forceinline__ uint32_t pack_half(float a, float b)
{
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}

template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// f(s) = cap tanh(s / cap).  Up to this cap it is cap - 2 cap / (1 + e^2y), y = s / cap,
// with 2 y log2 e straight from the product: wrong by cap 1.4 2^-22 at most, 2e-5
// (weights are rounded to 2^-11).  The error grows with the cap, though, so that
// larger ones take capped(), which is some dozen instructions more a score (two pieces
// of 4,096 tokens against 12-16k positions, 8 x 4 heads of 128: 3,550 us with a cap of
// 1,000, 2,610 with one of 30).
constexpr float kPlainCap = 64.0f;
__device__ __forceinline__ bool plain_cap(const AttendArgs &a) { return a.softcap <= kPlainCap; }

// What a product is multiplied by: to 2 y log2 e for a plain cap, else to s log2 e.
__device__ __forceinline__ float score_multiplier(const AttendArgs &a, float scale)
{
    return a.softcap > 0.0f && plain_cap(a) ? scale * (2.0f * kLog2e) / a.softcap : scale * kLog2e;
}

// f of s = score log2 e, right relative to s: where |y| < 1/2 by the Taylor series of
// tanh y / y up to y^12 (the next term is below 2^-23), else as above, e^2y being away
// from 1.
__device__ __forceinline__ float capped_near(const AttendArgs &a, float s)
{
    const float y = s * a.cap_inv, w = y * y;
    float t = 21844.0f / 6081075.0f;
    t = fmaf(t, w, -1382.0f / 155925.0f);
    t = fmaf(t, w, 62.0f / 2835.0f);
    t = fmaf(t, w, -17.0f / 315.0f);
    t = fmaf(t, w, 2.0f / 15.0f);
    t = fmaf(t, w, -1.0f / 3.0f);
    return fmaf(s * w, t, s);
}
__device__ __forceinline__ float capped(const AttendArgs &a, float s)
{
    const float y = s * a.cap_inv;
    const float far = fmaf(-2.0f * a.cap2, __fdividef(1.0f, 1.0f + ex2(y * (2.0f * kLog2e))), a.cap2);
    return fabsf(y) < 0.5f ? capped_near(a, s) : far;
}

// The sum of weights counts a page's at kRef / vs.  With scales from 2^-100 on
// that is at most 2^80, and 2^30 weights of 2^15 add up to less than float32
// holds; the share of a scale of 2^100 is 2^-120, so that one such page is not
// lost either.
constexpr float kRef = 0x1p-20f, kLog2Ref = -20.0f;
__device__ __forceinline__ float value_scale(float vs) { return fmaxf(vs, FKV_PAGE_MIN_SCALE); }
__device__ __forceinline__ float share_of(float vs) { return __fdividef(kRef, vs); }

}  // namespace fkvd

// Rows of 256 (attend_prompt.cu): a.row_tiles, splits and chunk as for the steps.
int prompt_rows();
cudaError_t launch_attend_prompt(const fkv_ctx *ctx, const fkvd::AttendArgs &a, int dim, int format, int dtype,
                                 cudaStream_t st);
