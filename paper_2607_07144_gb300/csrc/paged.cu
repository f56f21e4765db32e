// The paged 8-bit K/V cache: block tables and slot maps from request lengths
// (k_page_plan), quantising writes (k_page_write) and the way back to a K/V
// cache (k_page_read).  Attention over the pages is in attend.cu.
#include <type_traits>

#include "paged.cuh"

using namespace fkvd;

namespace {

// ------------------------------------------------------------------ plan --
// Every block scans the requests (tokens, pages needed, pages given back; a
// consecutive share a thread) and then does its part of the pages and of the
// token rows from the inputs alone: a page given back in the call is looked up
// where its request's table has it, not on the stack.  So blocks wait for one
// another nowhere, and share no counter that overlapping calls or graphs would
// share too.  Only what may be the inputs' own arrays, the lengths and the count,
// has to come after: in the same block where one block does the call (up to 4096
// rows), else in a second launch of one block, whose own scan runs while the
// first launch does.  Latency bounds both: a chain of three or four loads.
constexpr int kPlanThreads = 1024, kPlanRows = 4;      // rows a thread
constexpr int kPlanSmem = FKV_PAGE_MAX_REQ * 3 * sizeof(int);

struct PlanArgs {
    const int *n_new, *kv_len, *taken;
    int *table, *free_ids, *cu, *positions, *kv_len_out, *taken_out;
    int64_t *slots;
    int64_t table_stride, n_free, rows;
    int n_req, width, block, share;
    FastDiv div;
    unsigned *status;
};

__device__ __forceinline__ int blocks_of(const PlanArgs &a, int tokens)
{
    return static_cast<int>(a.div.div(static_cast<unsigned>(tokens) + a.block - 1));
}

// The last i < n with first[i] <= x (first[0] <= x).
__device__ __forceinline__ int last_from(const int *first, int n, int x)
{
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid] <= x)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}

// What a call amounts to; all or nothing: one that does not fit has no tokens
// and no pages.
struct PlanTotals {
    int tokens, pages, back;
    int taken0, taken1;
    bool bad;
};

// The requests' totals, and (cu not null) the sums before every request: n_req
// each in cu, need and back.  Latency bounds a plan: a scan of the requests and
// chains of two or three loads (64 requests, a token each, 7 us, 500 with 461k
// tokens 13).
__device__ PlanTotals plan_scan(const PlanArgs &a, int *cu, int *need, int *back)
{
    __shared__ int part[3][32];
    __shared__ int bad_s;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int r0 = min(tid * a.share, a.n_req), r1 = min(r0 + a.share, a.n_req);
    PlanTotals p;
    p.taken0 = *a.taken;
    if (tid == 0)
        bad_s = 0;
    __syncthreads();
    auto count = [&](int r, int *v) {
        const int nn = a.n_new[r], len = a.kv_len[r];
        v[0] = v[1] = v[2] = 0;
        if (len < 0 || len > FKV_PAGE_MAX_LEN || nn > FKV_PAGE_MAX_LEN - len || blocks_of(a, len) > a.width)
            return false;
        if (nn < 0) {
            v[2] = blocks_of(a, len);
            return true;
        }
        const int nb = blocks_of(a, len + nn);
        v[0] = nn;
        v[1] = nb - blocks_of(a, len);
        return nb <= a.width;
    };
    // Sums are kept in 32 bits; one that does not fit makes the call one that does
    // not either.
    int sum[3];
    bool over = false;
    {
        long long wide[3] = {0, 0, 0};
        for (int r = r0; r < r1; ++r) {
            int v[3];
            if (!count(r, v))
                over = true;
#pragma unroll
            for (int c = 0; c < 3; ++c)
                wide[c] += v[c];
        }
#pragma unroll
        for (int c = 0; c < 3; ++c) {
            over |= wide[c] > 0x7fffffffll;
            sum[c] = static_cast<int>(min(wide[c], 0x7fffffffll));
        }
    }
    // whether a warp's values, each below 2^31, sum to less than that
    auto fits = [](unsigned x) {
        const long long hi = __reduce_add_sync(~0u, x >> 15), lo = __reduce_add_sync(~0u, x & 0x7fffu);
        return (hi << 15) + lo <= 0x7fffffffll;
    };
    int before[3], all[3];
#pragma unroll
    for (int c = 0; c < 3; ++c) {
        over |= !fits(sum[c]);
        int x = sum[c];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(~0u, x, o);
            if (lane >= o)
                x += y;
        }
        if (lane == 31)
            part[c][warp] = x;
        before[c] = x - sum[c];
    }
    if (over)
        bad_s = 1;
    __syncthreads();
    over = bad_s;
#pragma unroll
    for (int c = 0; c < 3; ++c) {
        int x = part[c][lane];
        over |= !fits(x);
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(~0u, x, o);
            if (lane >= o)
                x += y;
        }
        const int prev = __shfl_sync(~0u, x, warp > 0 ? warp - 1 : 0);
        before[c] += warp > 0 ? prev : 0;
        all[c] = __shfl_sync(~0u, x, 31);
    }
    const long long taken1 = static_cast<long long>(p.taken0) - all[2];
    p.bad = over || p.taken0 < 0 || p.taken0 > a.n_free || taken1 < 0 || taken1 + all[1] > a.n_free || all[0] > a.rows;
    p.taken1 = p.bad ? p.taken0 : static_cast<int>(taken1);
    p.tokens = p.bad ? 0 : all[0];
    p.pages = p.bad ? 0 : all[1];
    p.back = p.bad ? 0 : all[2];
    if (cu) {
        for (int r = r0; r < r1; ++r) {
            cu[r] = p.bad ? 0 : before[0];
            need[r] = p.bad ? 0 : before[1];
            back[r] = p.bad ? 0 : before[2];
            if (r + 1 < r1) {
                int v[3];
                count(r, v);
#pragma unroll
                for (int c = 0; c < 3; ++c)
                    before[c] += v[c];
            }
        }
        __syncthreads();
    }
    return p;
}

// What may lie over the inputs: lengths and count.
__device__ __forceinline__ void plan_finish(const PlanArgs &a, const PlanTotals &p)
{
    for (int r = threadIdx.x; r < a.n_req; r += kPlanThreads) {
        const int nn = a.n_new[r], len = a.kv_len[r];
        a.kv_len_out[r] = p.bad ? len : (nn < 0 ? 0 : len + nn);
    }
    if (threadIdx.x == 0) {
        *a.taken_out = p.taken1 + p.pages;
        if (p.bad)
            atomicOr(a.status, FKV_ST_RANGE);
    }
}

__global__ void __launch_bounds__(kPlanThreads) k_page_plan(PlanArgs a)
{
    extern __shared__ int sums[];            // n_req sums each of tokens, pages needed and pages given back
    int *const cu = sums, *const need = sums + a.n_req, *const back = need + a.n_req;
    const PlanTotals p = plan_scan(a, cu, need, back);
    // of all the launch's threads
    const int gtid = static_cast<int>(blockIdx.x) * kPlanThreads + threadIdx.x, gsize = static_cast<int>(gridDim.x) * kPlanThreads;

    // the x-th page that comes back, and the x-th that is taken: off the stack
    // once those that came back are used up
    auto returned = [&](int x) {
        const int r = last_from(back, a.n_req, x);
        return a.table[r * a.table_stride + x - back[r]];
    };
    auto fresh = [&](int x) { return x < p.back ? returned(x) : a.free_ids[p.taken1 + x]; };

    // the thread's first page of either kind: on their way while the rows are
    // looked up
    int page = 0, page_r = 0, page_len = 0, page_back = 0;
    if (gtid < p.pages) {
        page_r = last_from(need, a.n_req, gtid);
        page = fresh(gtid);
        page_len = a.kv_len[page_r];
    }
    if (gtid < p.back)
        page_back = returned(gtid);
    for (int r = gtid; r <= a.n_req; r += gsize)
        a.cu[r] = r < a.n_req ? cu[r] : p.tokens;
    // the rows, whose loads are in flight together
    for (int64_t t0 = gtid; t0 < a.rows; t0 += static_cast<int64_t>(kPlanRows) * gsize) {
        int id[kPlanRows], pos[kPlanRows];
#pragma unroll
        for (int k = 0; k < kPlanRows; ++k) {
            const int64_t t = t0 + static_cast<int64_t>(k) * gsize;
            id[k] = pos[k] = -1;
            if (t < p.tokens) {
                const int r = last_from(cu, a.n_req, static_cast<int>(t)), len = a.kv_len[r], had = blocks_of(a, len);
                pos[k] = len + static_cast<int>(t) - cu[r];
                const int j = static_cast<int>(a.div.div(pos[k]));
                id[k] = j < had ? a.table[r * a.table_stride + j] : fresh(need[r] + j - had);
            }
        }
#pragma unroll
        for (int k = 0; k < kPlanRows; ++k) {
            const int64_t t = t0 + static_cast<int64_t>(k) * gsize;
            if (t < a.rows) {
                const int off = pos[k] - static_cast<int>(a.div.div(pos[k])) * a.block;
                a.slots[t] = id[k] < 0 ? -1 : static_cast<int64_t>(id[k]) * a.block + off;
                a.positions[t] = pos[k];
            }
        }
    }
    if (gtid < p.pages)
        a.table[page_r * a.table_stride + blocks_of(a, page_len) + gtid - need[page_r]] = page;
    if (gtid < p.back)
        a.free_ids[p.taken1 + gtid] = page_back;
    for (int i = gtid + gsize; i < p.pages; i += gsize) {
        const int r = last_from(need, a.n_req, i), id = fresh(i);
        a.table[r * a.table_stride + blocks_of(a, a.kv_len[r]) + i - need[r]] = id;
    }
    for (int i = gtid + gsize; i < p.back; i += gsize)
        a.free_ids[p.taken1 + i] = returned(i);
    if (gridDim.x == 1) {
        __syncthreads();
        plan_finish(a, p);
    }
}

__global__ void __launch_bounds__(kPlanThreads) k_page_plan_finish(PlanArgs a)
{
    const PlanTotals p = plan_scan(a, nullptr, nullptr, nullptr);
    asm volatile("griddepcontrol.wait;" ::: "memory");     // no block reads the inputs from here on
    plan_finish(a, p);
}

// ----------------------------------------------------------------- write --
template <typename T> __device__ __forceinline__ void load16(const T *p, float *x);
template <> __device__ __forceinline__ void load16<float>(const float *p, float *x)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float4 v = reinterpret_cast<const float4 *>(p)[i];
        x[4 * i] = v.x, x[4 * i + 1] = v.y, x[4 * i + 2] = v.z, x[4 * i + 3] = v.w;
    }
}
template <> __device__ __forceinline__ void load16<__half>(const __half *p, float *x)
{
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint4 v = reinterpret_cast<const uint4 *>(p)[i];
        const __half2 *h = reinterpret_cast<const __half2 *>(&v);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float2 f = __half22float2(h[k]);
            x[8 * i + 2 * k] = f.x, x[8 * i + 2 * k + 1] = f.y;
        }
    }
}
template <> __device__ __forceinline__ void load16<__nv_bfloat16>(const __nv_bfloat16 *p, float *x)
{
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint4 v = reinterpret_cast<const uint4 *>(p)[i];
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            x[8 * i + 2 * k] = __uint_as_float(w[k] << 16);
            x[8 * i + 2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
        }
    }
}

__device__ __forceinline__ float finite_abs(float v)
{
    const float a = fabsf(v);
    return a <= 3.402823466e38f ? a : 0.0f;      // false for infinities and NaN
}

// The scale that brings amax into the format's range (fkv.h): e4m3 the smallest
// power of two, so that a later, larger scale rounds no stored code again but
// in the lowest (subnormal) ones; int8 amax / 127, which uses all its codes.  Either
// within [2^-100, 2^100].
template <int FMT> __device__ __forceinline__ float scale_of(float amax)
{
    if (FMT == FKV_INT8)
        return fminf(fmaxf(__fdiv_rn(amax, 127.0f), FKV_PAGE_MIN_SCALE), FKV_PAGE_MAX_SCALE);
    const uint32_t u = __float_as_uint(amax);
    // amax = 1.m 2^E; 448 = 1.75 2^8
    const int e = static_cast<int>(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u);
    return __uint_as_float(static_cast<uint32_t>(min(max(e, -100), 100) + 127) << 23);
}

// 16 values times inv, rounded to codes.
template <int FMT> __device__ __forceinline__ uint4 codes16(const float *x, float inv)
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float a = x[4 * i] * inv, b = x[4 * i + 1] * inv, c = x[4 * i + 2] * inv, d = x[4 * i + 3] * inv;
        if (FMT == FKV_INT8) {
            int q[4];
            const float y[4] = {a, b, c, d};
#pragma unroll
            for (int k = 0; k < 4; ++k)       // NaN: 0 (the conversion's), infinities: +-127
                q[k] = max(-127, min(127, __float2int_rn(y[k])));
            w[i] = (q[0] & 255) | (q[1] & 255) << 8 | (q[2] & 255) << 16 | static_cast<uint32_t>(q[3]) << 24;
        } else {
            uint16_t lo, hi;
            asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
            asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
            w[i] = static_cast<uint32_t>(hi) << 16 | lo;
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// A NaN has no code a reader could take as one: it is stored as zero.
__device__ __forceinline__ bool drop_nan(float *x)
{
    bool any = false;
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (x[i] != x[i])
            x[i] = 0.0f, any = true;
    return any;
}

template <int FMT> __device__ __forceinline__ void values16(const uint4 &v, float *x)
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (FMT == FKV_INT8) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                x[4 * i + k] = static_cast<float>(static_cast<int8_t>(w[i] >> (8 * k)));
        } else {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float2 f = __half22float2(e4m3x2_half2(static_cast<uint16_t>(w[i] >> (16 * k))));
                x[4 * i + 2 * k] = f.x, x[4 * i + 2 * k + 1] = f.y;
            }
        }
    }
}

struct WriteArgs {
    uint8_t *pool[2];
    float *scale[2];
    const void *x[2];
    int64_t x_tok[2], x_head[2];
    const int64_t *slots;
    int64_t T, sb, sh, st, scb, sch, n_slots;              // n_slots: at most 2^32
    int block, stretch, heads;
    FastDiv by_block, by_heads;
    unsigned *status;
};

// 16 elements as they lie in memory.
template <typename T> struct Raw {
    uint4 v[sizeof(T)];
};

template <typename T> __device__ __forceinline__ Raw<T> load_raw(const T *p)
{
    Raw<T> r;
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(T)); ++i)
        r.v[i] = __ldg(reinterpret_cast<const uint4 *>(p) + i);
    return r;
}

// The largest magnitude of some elements, two at a time for 16-bit types; a NaN
// makes it NaN.
template <typename T> struct Largest {
    uint32_t m = 0;
    __device__ __forceinline__ void take(const Raw<T> &r)
    {
        const uint32_t *w = reinterpret_cast<const uint32_t *>(&r);
#pragma unroll
        for (int i = 0; i < 4 * static_cast<int>(sizeof(T)); ++i) {
            if (std::is_same<T, float>::value)
                // magnitudes compare as integers do, NaN above infinity
                m = max(m, w[i] & 0x7fffffffu);
            else if (std::is_same<T, __half>::value)
                asm("max.NaN.f16x2 %0, %0, %1;" : "+r"(m) : "r"(w[i] & 0x7fff7fffu));
            else
                asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(w[i] & 0x7fff7fffu));
        }
    }
    __device__ __forceinline__ float value() const
    {
        if (std::is_same<T, float>::value)
            return __uint_as_float(m);
        if (std::is_same<T, __half>::value) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&m));
            return f.x != f.x || f.y != f.y ? __uint_as_float(0x7fffffffu) : fmaxf(f.x, f.y);
        }
        const uint32_t b = max(m & 0xffffu, m >> 16);
        return __uint_as_float(b << 16);
    }
};

// codes16 of values of at most the scale's range: no limits to look at, and an
// int8's rounding is an addition of 1.5 2^23, whose sum's low byte is the code.
template <int FMT> __device__ __forceinline__ uint4 codes16_inside(const float *x, float inv)
{
    if (FMT == FKV_E4M3) {
        return codes16<FMT>(x, inv);
    } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t q[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                q[k] = __float_as_uint(__fadd_rn(__fmul_rn(x[4 * i + k], inv), 12582912.0f));
            w[i] = __byte_perm(__byte_perm(q[0], q[1], 0x0040), __byte_perm(q[2], q[3], 0x0040), 0x5410);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// A run of tokens with consecutive slots inside one page belongs to the group of
// GT threads whose stretch of tokens holds its first one, for one head and K or
// V; the group reads and writes that page and its scale alone: no atomics, and
// the same result in any order of the groups.  A few tokens (a step's) get a
// warp each, many a block of 128 threads for as many tokens as a page holds,
// which keeps up to four rows a thread in registers between the search for the
// largest magnitude and the rounding (longer runs are read again).  Bytes bound
// long calls, the chain slot, page, store a step's.  9 prompts of 1,000 to 8,192
// tokens, 8 heads of 128, bf16 to int8: 59 us, 5.2 TB/s, from float32 150 us, 3.4
// TB/s (fewer warps, for its registers); 64 tokens, one a page: 5.7 us, the host's.
template <int D, int FMT, typename T, int GT> __global__ void __launch_bounds__(GT == 32 ? 256 : GT, GT == 32 || sizeof(T) == 4 ? 1 : 8) k_page_write(WriteArgs a)
{
    constexpr int C = D / 16, R = GT / C, KEEP = 4;        // 16-element pieces a row, rows at a time, kept of them
    __shared__ uint32_t red[GT / 32];
    const int lane = threadIdx.x & 31, tid = GT == 32 ? lane : threadIdx.x, c = tid % C, row0 = tid / C;
    unsigned item = blockIdx.x;
    if (GT == 32)
        item = item * 8 + (threadIdx.x >> 5);
    const unsigned both = a.by_heads.div(item);
    const int h = static_cast<int>(item - both * a.heads), kv = both & 1;
    const int64_t t0 = static_cast<int64_t>(both >> 1) * a.stretch;
    if (t0 >= a.T)
        return;
    const int64_t t1 = min(t0 + a.stretch, a.T);
    const T *const x = static_cast<const T *>(a.x[kv]) + h * a.x_head[kv] + c * 16;
    bool nan = false, range = false;
    for (int64_t base = t0; base < t1; base += 32) {
        // a lane a token: which of them begin a run (every warp of a group finds the same)
        const int64_t mine = base + lane;
        int64_t slot_l = -1;
        bool lead = false;
        if (mine < t1) {
            slot_l = a.slots[mine];
            const int64_t prev = mine > 0 ? a.slots[mine - 1] : -2;
            if (slot_l >= a.n_slots)
                range = true;
            else if (slot_l >= 0)
                lead = prev != slot_l - 1 || slot_l == static_cast<int64_t>(a.by_block.div(static_cast<unsigned>(slot_l))) * a.block;
        }
        unsigned leads = __ballot_sync(~0u, lead);
        while (leads) {
            const int who = __ffs(leads) - 1;
            leads &= leads - 1;
            const int64_t t = base + who, slot = __shfl_sync(~0u, slot_l, who), blk = a.by_block.div(static_cast<unsigned>(slot));
            const int off = static_cast<int>(slot - blk * a.block);
            // the run's length: consecutive slots up to the page's end
            const int most = static_cast<int>(min(static_cast<int64_t>(a.block - off), a.T - t));
            // a block loads the run's rows before it knows the length, as if it were as
            // long as the page allows (a step's are mostly one row)
            Raw<T> keep[KEEP];
#pragma unroll
            for (int k = 0; k < KEEP; ++k)
                if ((GT > 32 || k == 0) && row0 + k * R < most)
                    keep[k] = load_raw<T>(x + (t + row0 + k * R) * a.x_tok[kv]);
            int len = most;
            for (int i = 0; i < most; i += 32) {
                const unsigned off_run = __ballot_sync(~0u, i + lane < most && a.slots[t + i + lane] != slot + i + lane);
                if (off_run) {
                    len = i + __ffs(off_run) - 1;
                    break;
                }
            }
            float *const sp = a.scale[kv] + blk * a.scb + h * a.sch;
            const float was = off > 0 ? *sp : 0.0f;
            uint8_t *const page = a.pool[kv] + blk * a.sb + h * a.sh + c * 16;
            if (GT == 32) {
#pragma unroll
                for (int k = 1; k < KEEP; ++k)
                    if (row0 + k * R < len)
                        keep[k] = load_raw<T>(x + (t + row0 + k * R) * a.x_tok[kv]);
            }
            Largest<T> most_v;
#pragma unroll
            for (int k = 0; k < KEEP; ++k)
                if (row0 + k * R < len)
                    most_v.take(keep[k]);
            for (int i = row0 + KEEP * R; i < len; i += R)
                most_v.take(load_raw<T>(x + (t + i) * a.x_tok[kv]));
            // as integers: magnitudes, a NaN above all
            uint32_t amax_u = __float_as_uint(most_v.value());
            auto join = [&]() {
                amax_u = __reduce_max_sync(~0u, amax_u);
                if (GT > 32) {
                    __syncthreads();       // red is free (also: every thread has read the page's old scale)
                    if (lane == 0)
                        red[threadIdx.x >> 5] = amax_u;
                    __syncthreads();
#pragma unroll
                    for (int w = 0; w < GT / 32; ++w)
                        amax_u = max(amax_u, red[w]);
                }
            };
            join();
            // infinities or NaN among the values, or some beyond the largest code of the
            // largest scale (of int8; e4m3's, 448, is larger)
            const bool odd = amax_u > __float_as_uint(127.0f * FKV_PAGE_MAX_SCALE);
            if (odd) {
                // rare: the largest finite magnitude
                float amax = 0.0f;
                for (int i = row0; i < len; i += R) {
                    float v[16];
                    load16<T>(x + (t + i) * a.x_tok[kv], v);
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        amax = fmaxf(amax, finite_abs(v[e]));
                }
                amax_u = __float_as_uint(amax);
                join();
            }
            const float want = amax_u ? scale_of<FMT>(__uint_as_float(amax_u)) : FKV_PAGE_MIN_SCALE;
            // a page's scale never shrinks while it has rows
            const float now = was >= want ? was : want;
            const float inv = __frcp_rn(now);
            if (!odd) {
#pragma unroll
                for (int k = 0; k < KEEP; ++k)
                    if (row0 + k * R < len) {
                        float v[16];
                        load16<T>(reinterpret_cast<const T *>(&keep[k]), v);
                        *reinterpret_cast<uint4 *>(page + (off + row0 + k * R) * a.st) = codes16_inside<FMT>(v, inv);
                    }
            }
            for (int i = odd ? row0 : row0 + KEEP * R; i < len; i += R) {
                float v[16];
                load16<T>(x + (t + i) * a.x_tok[kv], v);
                nan |= drop_nan(v);
                *reinterpret_cast<uint4 *>(page + (off + i) * a.st) = codes16<FMT>(v, inv);
            }
            __syncwarp();
            if (now != was) {
                const float ratio = __fmul_rn(was, inv);
                for (int i = row0; i < off; i += R) {
                    uint4 *p = reinterpret_cast<uint4 *>(page + i * a.st);
                    float v[16];
                    values16<FMT>(*p, v);
                    *p = codes16<FMT>(v, ratio);
                }
                if (tid == 0)
                    *sp = now;
            }
        }
    }
    if (nan)
        atomicOr(a.status, FKV_ST_CORRUPT);
    if (range)
        atomicOr(a.status, FKV_ST_RANGE);
}

// ------------------------------------------------------------------ read --
template <typename T> __device__ __forceinline__ void store16(T *p, const float *x);
template <> __device__ __forceinline__ void store16<float>(float *p, const float *x)
{
#pragma unroll
    for (int i = 0; i < 4; ++i)
        reinterpret_cast<float4 *>(p)[i] = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
}
template <> __device__ __forceinline__ void store16<__half>(__half *p, const float *x)
{
    __half2 h[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
        h[i] = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
    reinterpret_cast<uint4 *>(p)[0] = *reinterpret_cast<uint4 *>(&h[0]);
    reinterpret_cast<uint4 *>(p)[1] = *reinterpret_cast<uint4 *>(&h[4]);
}
template <> __device__ __forceinline__ void store16<__nv_bfloat16>(__nv_bfloat16 *p, const float *x)
{
    __nv_bfloat162 h[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
        h[i] = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    reinterpret_cast<uint4 *>(p)[0] = *reinterpret_cast<uint4 *>(&h[0]);
    reinterpret_cast<uint4 *>(p)[1] = *reinterpret_cast<uint4 *>(&h[4]);
}

struct ReadArgs {
    const uint8_t *pool[2];
    const float *scale[2];
    void *out[2];
    int64_t o_batch[2], o_head[2], o_pos[2];
    const int *kv_len, *table;
    int64_t table_stride, t0, t1, sb, sh, st, scb, sch, n_blocks;
    int n_req, width, block, heads, units, kv0;
    FastDiv div;
    unsigned *status;
};

// A warp per 16 positions of one page, head and K or V: 16 bytes of codes a
// lane and step, their 16 values out.  A call moves D + 1 .. 4 D bytes a
// vector and computes next to nothing: the bytes bound it (4 sequences of 9-33k
// positions, 8 heads of 128, e4m3 to bf16: 93 us, 6.2 TB/s).
template <int D, int FMT, typename T> __global__ void __launch_bounds__(256) k_page_read(ReadArgs a)
{
    constexpr int C = D / 16, R = 32 / C;
    const int lane = threadIdx.x & 31, c = lane % C;
    const int64_t unit = static_cast<int64_t>(blockIdx.x) * 8 + (threadIdx.x >> 5);
    const int r = static_cast<int>(unit / a.units), u = static_cast<int>(unit - static_cast<int64_t>(r) * a.units);
    const int h = blockIdx.y, kv = a.kv0 + blockIdx.z;
    if (r >= a.n_req)
        return;
    const int len = a.kv_len[r];
    const int64_t p0 = (a.t0 / 16 + u) * 16;
    const int64_t to = min(a.t1, static_cast<int64_t>(len));
    if (p0 >= to)
        return;
    const int j = static_cast<int>(a.div.div(static_cast<unsigned>(p0)));
    int id = -1;
    if (j < a.width)
        id = a.table[r * a.table_stride + j];
    if (id < 0 || id >= a.n_blocks) {
        if (lane == 0)
            atomicOr(a.status, FKV_ST_RANGE);
        return;
    }
    const float s = a.scale[kv][id * a.scb + h * a.sch];
    const uint8_t *page = a.pool[kv] + id * a.sb + h * a.sh + (p0 - static_cast<int64_t>(j) * a.block) * a.st + c * 16;
    T *out = static_cast<T *>(a.out[kv]) + r * a.o_batch[kv] + h * a.o_head[kv] + p0 * a.o_pos[kv] + c * 16;
#pragma unroll
    for (int i = lane / C; i < 16; i += R) {
        if (p0 + i < a.t0 || p0 + i >= to)
            continue;
        float v[16];
        values16<FMT>(*reinterpret_cast<const uint4 *>(page + i * a.st), v);
#pragma unroll
        for (int k = 0; k < 16; ++k)
            v[k] *= s;
        store16<T>(out + i * a.o_pos[kv], v);
    }
}

template <int D, int FMT, typename T> cudaError_t write_by(const WriteArgs &a, int64_t items, cudaStream_t st)
{
    if (a.stretch == 1)
        k_page_write<D, FMT, T, 32><<<static_cast<unsigned>((items + 7) / 8), 256, 0, st>>>(a);
    else
        k_page_write<D, FMT, T, 128><<<static_cast<unsigned>(items), 128, 0, st>>>(a);
    return cudaGetLastError();
}

template <int FMT, typename T> cudaError_t write_as(const WriteArgs &a, int dim, cudaStream_t st)
{
    const int64_t items = (a.T + a.stretch - 1) / a.stretch * 2 * a.heads;
    return dim == 64 ? write_by<64, FMT, T>(a, items, st) : write_by<128, FMT, T>(a, items, st);
}

template <int FMT, typename T> cudaError_t read_as(const ReadArgs &a, int dim, dim3 grid, cudaStream_t st)
{
    if (dim == 64)
        k_page_read<64, FMT, T><<<grid, 256, 0, st>>>(a);
    else
        k_page_read<128, FMT, T><<<grid, 256, 0, st>>>(a);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_page_plan(const fkv_ctx *ctx, const fkv_plan &p, cudaStream_t st)
{
    PlanArgs a;
    a.n_new = p.n_new, a.kv_len = p.kv_len, a.taken = p.taken;
    a.table = p.table, a.free_ids = p.free, a.cu = p.cu, a.positions = p.pos;
    a.kv_len_out = p.kv_len_out, a.taken_out = p.taken_out, a.slots = p.slots;
    a.table_stride = p.table_stride, a.n_free = p.n_free, a.rows = p.rows;
    a.n_req = static_cast<int>(p.n_req), a.width = static_cast<int>(p.width), a.block = static_cast<int>(p.block);
    a.div = FastDiv::make(static_cast<unsigned>(p.block));
    a.status = ctx->d_status;
    a.share = (a.n_req + kPlanThreads - 1) / kPlanThreads;
    const int64_t per = kPlanThreads * kPlanRows, want = (a.rows + per - 1) / per;
    // a block an SM at most; each scans all requests
    const int blocks = static_cast<int>(want < 1 ? 1 : want < ctx->sms ? want : ctx->sms);
    const size_t smem = static_cast<size_t>(a.n_req) * 3 * sizeof(int);
    cudaError_t e = kernel_use(ctx, reinterpret_cast<const void *>(k_page_plan), kPlanThreads, kPlanSmem, nullptr);
    if (e != cudaSuccess)
        return e;
    k_page_plan<<<blocks, kPlanThreads, smem, st>>>(a);
    e = cudaGetLastError();
    if (e != cudaSuccess || blocks == 1)
        return e;
    return launch_after(k_page_plan_finish, 1, kPlanThreads, 0, st, a);
}

cudaError_t launch_page_write(const fkv_ctx *ctx, const fkv_pages *p, const fkv_rows *k, const fkv_rows *v,
                              const int64_t *slots, int64_t T, cudaStream_t st)
{
    WriteArgs a;
    const fkv_rows *x[2] = {k, v};
    for (int i = 0; i < 2; ++i) {
        a.pool[i] = static_cast<uint8_t *>(i ? p->v : p->k);
        a.scale[i] = i ? p->v_scale : p->k_scale;
        a.x[i] = x[i]->data;
        a.x_tok[i] = x[i]->stride_tok;
        a.x_head[i] = x[i]->stride_head;
    }
    a.slots = slots, a.T = T;
    a.sb = p->stride_block, a.sh = p->stride_head, a.st = p->stride_pos;
    a.scb = p->scale_stride_block, a.sch = p->scale_stride_head;
    a.n_slots = p->n_blocks * p->block, a.block = p->block;
    a.status = ctx->d_status;
    // a warp a token while that fills the device up to a few times over, else a
    // block for as many tokens as a page holds (8 heads of 128: 64 tokens one a page
    // 6 us against 32 as blocks, 600 such 10 against 33, 1,200 17 against 35; 600 of two
    // prompts 12 against 6, 1,200 of them 16 against 6.5: large calls are prompts mostly)
    a.heads = p->n_heads;
    a.by_block = FastDiv::make(static_cast<unsigned>(p->block)), a.by_heads = FastDiv::make(static_cast<unsigned>(p->n_heads));
    a.stretch = T * p->n_heads * 2 <= static_cast<int64_t>(ctx->sms) * 64 ? 1 : p->block;
    const bool i8 = p->format == FKV_INT8;
    switch (k->dtype) {
    case FKV_F32:
        return i8 ? write_as<FKV_INT8, float>(a, p->dim, st) : write_as<FKV_E4M3, float>(a, p->dim, st);
    case FKV_F16:
        return i8 ? write_as<FKV_INT8, __half>(a, p->dim, st) : write_as<FKV_E4M3, __half>(a, p->dim, st);
    default:
        return i8 ? write_as<FKV_INT8, __nv_bfloat16>(a, p->dim, st) : write_as<FKV_E4M3, __nv_bfloat16>(a, p->dim, st);
    }
}

cudaError_t launch_page_read(const fkv_ctx *ctx, const fkv_pages *p, const int32_t *kv_len, int64_t n_req,
                             const int32_t *table, int64_t table_stride, int64_t width, int64_t t0, int64_t t1,
                             int64_t layer, const fkv_cache *k_out, const fkv_cache *v_out, cudaStream_t st)
{
    ReadArgs a;
    const fkv_cache *o[2] = {k_out, v_out};
    int dtype = 0;
    for (int i = 0; i < 2; ++i) {
        a.pool[i] = static_cast<const uint8_t *>(i ? p->v : p->k);
        a.scale[i] = i ? p->v_scale : p->k_scale;
        a.out[i] = nullptr;
        if (o[i]) {
            dtype = o[i]->dtype;
            const int64_t esz = dtype == FKV_F32 ? 4 : 2;
            a.out[i] = static_cast<uint8_t *>(o[i]->data) + layer * o[i]->stride_layer * esz;
            a.o_batch[i] = o[i]->stride_batch, a.o_head[i] = o[i]->stride_head, a.o_pos[i] = o[i]->stride_pos;
        }
    }
    a.kv_len = kv_len, a.table = table, a.table_stride = table_stride, a.t0 = t0, a.t1 = t1;
    a.sb = p->stride_block, a.sh = p->stride_head, a.st = p->stride_pos;
    a.scb = p->scale_stride_block, a.sch = p->scale_stride_head, a.n_blocks = p->n_blocks;
    a.n_req = static_cast<int>(n_req), a.width = static_cast<int>(width), a.block = p->block, a.heads = p->n_heads;
    a.div = FastDiv::make(p->block);
    a.status = ctx->d_status;
    a.units = static_cast<int>((t1 + 15) / 16 - t0 / 16);
    a.kv0 = k_out ? 0 : 1;
    const dim3 grid(static_cast<unsigned>((n_req * a.units + 7) / 8), p->n_heads, k_out && v_out ? 2 : 1);
    const bool i8 = p->format == FKV_INT8;
    switch (dtype) {
    case FKV_F32:
        return i8 ? read_as<FKV_INT8, float>(a, p->dim, grid, st) : read_as<FKV_E4M3, float>(a, p->dim, grid, st);
    case FKV_F16:
        return i8 ? read_as<FKV_INT8, __half>(a, p->dim, grid, st) : read_as<FKV_E4M3, __half>(a, p->dim, grid, st);
    default:
        return i8 ? read_as<FKV_INT8, __nv_bfloat16>(a, p->dim, grid, st)
                  : read_as<FKV_E4M3, __nv_bfloat16>(a, p->dim, grid, st);
    }
}
