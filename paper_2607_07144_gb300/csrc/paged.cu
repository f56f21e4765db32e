// The paged 8-bit K/V cache: block tables and slot maps from request lengths
// (k_page_plan), quantising writes (k_page_write) and the way back to a K/V
// cache (k_page_read).  Attention over the pages is in attend.cu.
#include <cooperative_groups.h>

#include "paged.cuh"

namespace cg = cooperative_groups;
using namespace fkvd;

namespace {

// ------------------------------------------------------------------ plan --
// One cluster of 8 blocks does a whole call: every block scans its share of
// the requests (tokens, blocks that come back, blocks needed), the shares'
// totals are exchanged through distributed shared memory, and the tokens are
// then spread over all threads, each finding its request by a binary search
// over the shares' prefix sums where they lie.  A second launch, or a grid-wide
// counter in a workspace that two graphs could share, is not needed; what
// bounds the call is the chain scan, exchange, exchange, store.
constexpr int kPlanBlocks = 8, kPlanThreads = 512;
constexpr int kPlanShare = FKV_PAGE_MAX_REQ / kPlanBlocks;   // requests a block can hold

struct PlanSmem {
    int cu[kPlanShare + 1];     // tokens before request i of this block's share
    int need[kPlanShare + 1];   // new blocks before it
    int back[kPlanShare + 1];   // returned blocks before it
    long long tot[3];           // the share's totals
    int warp[3][kPlanThreads / 32];
    int carry[3];
    int bad;                    // a length or the table's width does not fit
};

struct PlanArgs {
    const int *n_new, *kv_len, *taken;
    int *table, *free_ids, *cu, *positions, *kv_len_out, *taken_out;
    int64_t *slots;
    int64_t table_stride, n_free, rows;
    int n_req, width, block;
    FastDiv div;
    unsigned *status;
};

__device__ __forceinline__ int blocks_of(const PlanArgs &a, int tokens)
{
    return static_cast<int>(a.div.div(static_cast<unsigned>(tokens) + a.block - 1));
}

__global__ void __cluster_dims__(kPlanBlocks, 1, 1) __launch_bounds__(kPlanThreads) k_page_plan(PlanArgs a)
{
    extern __shared__ __align__(16) uint8_t raw[];
    PlanSmem &s = *reinterpret_cast<PlanSmem *>(raw);
    cg::cluster_group cluster = cg::this_cluster();
    const int me = cluster.block_rank(), tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int share = (a.n_req + kPlanBlocks - 1) / kPlanBlocks;
    const int r0 = min(me * share, a.n_req), r1 = min(r0 + share, a.n_req);
    if (tid == 0) {
        s.bad = 0;
        s.carry[0] = s.carry[1] = s.carry[2] = 0;
        s.tot[0] = s.tot[1] = s.tot[2] = 0;
    }
    const int taken0 = *a.taken;
    __syncthreads();

    // this share's exclusive sums, kPlanThreads requests at a time
    for (int base = r0; base < r1; base += kPlanThreads) {
        const int r = base + tid;
        int v[3] = {0, 0, 0};
        if (r < r1) {
            const int nn = a.n_new[r], len = a.kv_len[r];
            // 2^30: sums of a block's width stay inside 31 bits
            if (len < 0 || nn > (1 << 30) || len > (1 << 30) || blocks_of(a, max(len, 0)) > a.width) {
                s.bad = 1;
            } else if (nn < 0) {
                v[2] = blocks_of(a, len);
            } else {
                const int nb = blocks_of(a, len + nn);
                if (nb > a.width)
                    s.bad = 1;
                v[0] = nn;
                v[1] = nb - blocks_of(a, len);
            }
        }
        int inc[3];
#pragma unroll
        for (int c = 0; c < 3; ++c) {
            int x = v[c];
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(~0u, x, o);
                if (lane >= o)
                    x += y;
            }
            inc[c] = x;
            if (lane == 31)
                s.warp[c][warp] = x;
            // a share's tokens and blocks are counted in 64 bits beside the 32-bit prefix sums
            long long w = v[c];
#pragma unroll
            for (int o = 16; o; o >>= 1)
                w += __shfl_xor_sync(~0u, w, o);
            if (lane == 0 && w)
                atomicAdd(reinterpret_cast<unsigned long long *>(&s.tot[c]), static_cast<unsigned long long>(w));
        }
        __syncthreads();
        int pre[3];
#pragma unroll
        for (int c = 0; c < 3; ++c) {
            int x = s.carry[c];
            for (int w = 0; w < warp; ++w)
                x += s.warp[c][w];
            pre[c] = x + inc[c] - v[c];
        }
        if (r < r1) {
            s.cu[r - r0] = pre[0];
            s.need[r - r0] = pre[1];
            s.back[r - r0] = pre[2];
        }
        __syncthreads();
        if (tid == kPlanThreads - 1) {
#pragma unroll
            for (int c = 0; c < 3; ++c)
                s.carry[c] = pre[c] + v[c];
        }
        __syncthreads();
    }
    cluster.sync();

    // every block's totals: what lies before this share, and the whole call's
    long long before[3] = {0, 0, 0}, all[3] = {0, 0, 0};
    int first_tok[kPlanBlocks + 1];
    int bad = 0;
#pragma unroll
    for (int b = 0; b < kPlanBlocks; ++b) {
        const PlanSmem *o = cluster.map_shared_rank(&s, b);
        bad |= o->bad;
#pragma unroll
        for (int c = 0; c < 3; ++c) {
            const long long t = o->tot[c];
            if (b < me)
                before[c] += t;
            if (c == 0)
                first_tok[b] = static_cast<int>(min(all[0], 0x7fffffffll));
            all[c] += t;
        }
    }
    first_tok[kPlanBlocks] = static_cast<int>(min(all[0], 0x7fffffffll));
    const long long taken1 = taken0 - all[2];
    // all or nothing: a call that does not fit leaves lengths, table and stack as they are
    if (taken0 < 0 || taken0 > a.n_free || taken1 < 0 || taken1 + all[1] > a.n_free || all[0] > a.rows)
        bad = 1;
    const int64_t gtid = static_cast<int64_t>(me) * kPlanThreads + tid, gsize = kPlanBlocks * kPlanThreads;

    // blocks that come back go onto the stack before any is taken from it.  The
    // lengths' new values wait until every thread has read the old ones: the
    // outputs may be the inputs' own arrays.
    if (!bad) {
        for (int r = r0 + warp; r < r1; r += kPlanThreads / 32) {
            if (a.n_new[r] >= 0)
                continue;
            const int nb = blocks_of(a, a.kv_len[r]);
            const long long at = taken1 + before[2] + s.back[r - r0];
            for (int j = lane; j < nb; j += 32)
                a.free_ids[at + j] = a.table[r * a.table_stride + j];
        }
    }
    for (int r = r0 + tid; r < r1; r += kPlanThreads)
        a.cu[r] = bad ? 0 : static_cast<int>(before[0] + s.cu[r - r0]);
    if (gtid == 0)
        a.cu[a.n_req] = bad ? 0 : static_cast<int>(all[0]);
    cluster.sync();

    const int total = bad ? 0 : static_cast<int>(all[0]);
    for (int64_t t = gtid; t < a.rows; t += gsize) {
        int64_t slot = -1;
        int pos = -1;
        if (t < total) {
            int b = 0;
#pragma unroll
            for (int i = 1; i < kPlanBlocks; ++i)
                b += first_tok[i] <= t;
            // a share without tokens starts where the next one does: the last
            // share whose first token is t or before holds it
            const PlanSmem *o = cluster.map_shared_rank(&s, b);
            const int o0 = min(b * share, a.n_req), on = min(o0 + share, a.n_req) - o0;
            const int rel = static_cast<int>(t) - first_tok[b];
            int lo = 0, hi = on;          // the last request whose first token is rel or before
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (o->cu[mid] <= rel)
                    lo = mid;
                else
                    hi = mid;
            }
            const int r = o0 + lo, len = a.kv_len[r];
            pos = len + rel - o->cu[lo];
            const int j = static_cast<int>(a.div.div(pos)), off = pos - j * a.block, had = blocks_of(a, len);
            int id;
            if (j < had) {
                id = a.table[r * a.table_stride + j];
            } else {
                long long need0 = o->need[lo];
                for (int i = 0; i < b; ++i)
                    need0 += cluster.map_shared_rank(&s, i)->tot[1];
                id = a.free_ids[taken1 + need0 + j - had];
                if (off == 0 || rel == o->cu[lo])
                    a.table[r * a.table_stride + j] = id;
            }
            slot = id < 0 ? -1 : static_cast<int64_t>(id) * a.block + off;
        }
        a.slots[t] = slot;
        a.positions[t] = pos;
    }
    cluster.sync();
    // no block reads lengths, the taken count or another's shared memory from here on
    for (int r = r0 + tid; r < r1; r += kPlanThreads) {
        const int nn = a.n_new[r], len = a.kv_len[r];
        a.kv_len_out[r] = bad ? len : (nn < 0 ? 0 : len + nn);
    }
    if (gtid == 0) {
        *a.taken_out = bad ? taken0 : static_cast<int>(taken1 + all[1]);
        if (bad)
            atomicOr(a.status, FKV_ST_RANGE);
    }
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
// in the lowest (subnormal) ones; int8 amax / 127, which uses all its codes.
template <int FMT> __device__ __forceinline__ float scale_of(float amax)
{
    if (FMT == FKV_INT8)
        return fmaxf(__fdiv_rn(amax, 127.0f), FKV_PAGE_MIN_SCALE);
    const uint32_t u = __float_as_uint(amax);
    // amax = 1.m 2^E; 448 = 1.75 2^8
    const int e = static_cast<int>(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u);
    return e < -100 ? FKV_PAGE_MIN_SCALE : __uint_as_float(static_cast<uint32_t>(e + 127) << 23);
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
    int64_t T, sb, sh, st, scb, sch, n_blocks;
    int block, stretch;
    unsigned *status;
};

constexpr int kWriteThreads = 128;

// A block per (stretch of tokens, head, K or V).  A run of tokens with
// consecutive slots inside one page belongs to the block whose stretch holds
// its first token, which therefore reads and writes that page and its scale
// alone: no atomics, and the same result in any order of the blocks.  Bound by
// the bytes of long calls and by latency for a step's: a run is read for its
// largest magnitude, then read again (from L1) to be rounded.
template <int D, int FMT, typename T> __global__ void __launch_bounds__(kWriteThreads) k_page_write(WriteArgs a)
{
    constexpr int C = D / 16, R = kWriteThreads / C;       // 16-element chunks a row, rows at a time
    __shared__ float red[kWriteThreads / 32];
    __shared__ int len_s;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, c = tid % C, row0 = tid / C;
    const int kv = blockIdx.z, h = blockIdx.y;
    const int64_t t0 = static_cast<int64_t>(blockIdx.x) * a.stretch, t1 = min(t0 + a.stretch, a.T);
    const T *x = static_cast<const T *>(a.x[kv]) + h * a.x_head[kv] + c * 16;
    bool nan = false, range = false;
    for (int64_t t = t0; t < t1; ++t) {
        const int64_t slot = a.slots[t];
        if (slot < 0)
            continue;
        const int64_t blk = slot / a.block;
        const int off = static_cast<int>(slot - blk * a.block);
        if (t > 0 && off != 0 && a.slots[t - 1] == slot - 1)
            continue;
        if (blk >= a.n_blocks) {
            range = true;
            continue;
        }
        // the run's length: consecutive slots up to the page's end
        const int most = static_cast<int>(min(static_cast<int64_t>(a.block - off), a.T - t));
        if (tid == 0)
            len_s = most;
        __syncthreads();
        for (int i = tid; i < most; i += kWriteThreads)
            if (a.slots[t + i] != slot + i) {
                atomicMin(&len_s, i);
                break;
            }
        __syncthreads();
        const int len = len_s;
        float amax = 0.0f;
        for (int i = row0; i < len; i += R) {
            float v[16];
            load16<T>(x + (t + i) * a.x_tok[kv], v);
#pragma unroll
            for (int k = 0; k < 16; ++k)
                amax = fmaxf(amax, finite_abs(v[k]));
        }
#pragma unroll
        for (int o = 16; o; o >>= 1)
            amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, o));
        if (lane == 0)
            red[warp] = amax;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWriteThreads / 32; ++w)
            amax = fmaxf(amax, red[w]);
        float *sp = a.scale[kv] + blk * a.scb + h * a.sch;
        uint8_t *page = a.pool[kv] + blk * a.sb + h * a.sh + c * 16;
        const float want = amax > 0.0f ? scale_of<FMT>(amax) : FKV_PAGE_MIN_SCALE;
        const float was = off > 0 ? *sp : 0.0f;
        // a page's scale never shrinks while it has rows
        const float now = was >= want ? was : want;
        const float inv = __frcp_rn(now);
        for (int i = row0; i < len; i += R) {
            float v[16];
            load16<T>(x + (t + i) * a.x_tok[kv], v);
            nan |= drop_nan(v);
            *reinterpret_cast<uint4 *>(page + (off + i) * a.st) = codes16<FMT>(v, inv);
        }
        if (now != was) {
            const float ratio = __fmul_rn(was, inv);
            for (int i = row0; i < off; i += R) {
                uint4 *p = reinterpret_cast<uint4 *>(page + i * a.st);
                float v[16];
                values16<FMT>(*p, v);
                *p = codes16<FMT>(v, ratio);
            }
        }
        __syncthreads();       // every thread has read the old scale, red and len_s
        if (tid == 0)
            *sp = now;
    }
    if (nan)
        atomicOr(a.status, FKV_ST_CORRUPT);
    if (range && tid == 0)
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
// vector and computes next to nothing: the bytes bound it.
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

template <int FMT, typename T>
cudaError_t write_as(const fkv_ctx *ctx, const WriteArgs &a, int dim, dim3 grid, cudaStream_t st)
{
    (void)ctx;
    if (dim == 64)
        k_page_write<64, FMT, T><<<grid, kWriteThreads, 0, st>>>(a);
    else
        k_page_write<128, FMT, T><<<grid, kWriteThreads, 0, st>>>(a);
    return cudaGetLastError();
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

cudaError_t launch_page_plan(const fkv_ctx *ctx, const int32_t *n_new, const int32_t *kv_len, int64_t n_req,
                             int32_t *table, int64_t table_stride, int64_t width, int32_t *free_ids, int64_t n_free,
                             const int32_t *taken, int block, int32_t *cu, int64_t *slots, int32_t *positions,
                             int64_t rows, int32_t *kv_len_out, int32_t *taken_out, cudaStream_t st)
{
    PlanArgs a;
    a.n_new = n_new, a.kv_len = kv_len, a.taken = taken;
    a.table = table, a.free_ids = free_ids, a.cu = cu, a.positions = positions;
    a.kv_len_out = kv_len_out, a.taken_out = taken_out, a.slots = slots;
    a.table_stride = table_stride, a.n_free = n_free, a.rows = rows;
    a.n_req = static_cast<int>(n_req), a.width = static_cast<int>(width), a.block = block;
    a.div = FastDiv::make(block);
    a.status = ctx->d_status;
    const void *fn = reinterpret_cast<const void *>(k_page_plan);
    const cudaError_t e = kernel_use(ctx, fn, kPlanThreads, sizeof(PlanSmem), nullptr);
    if (e != cudaSuccess)
        return e;
    k_page_plan<<<kPlanBlocks, kPlanThreads, sizeof(PlanSmem), st>>>(a);
    return cudaGetLastError();
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
    a.n_blocks = p->n_blocks, a.block = p->block;
    a.status = ctx->d_status;
    // one token a block while that keeps the blocks to a few waves, else 16
    a.stretch = T * p->n_heads * 2 <= static_cast<int64_t>(ctx->sms) * 64 ? 1 : 16;
    const dim3 grid(static_cast<unsigned>((T + a.stretch - 1) / a.stretch), p->n_heads, 2);
    const bool i8 = p->format == FKV_INT8;
    switch (k->dtype) {
    case FKV_F32:
        return i8 ? write_as<FKV_INT8, float>(ctx, a, p->dim, grid, st) : write_as<FKV_E4M3, float>(ctx, a, p->dim, grid, st);
    case FKV_F16:
        return i8 ? write_as<FKV_INT8, __half>(ctx, a, p->dim, grid, st) : write_as<FKV_E4M3, __half>(ctx, a, p->dim, grid, st);
    default:
        return i8 ? write_as<FKV_INT8, __nv_bfloat16>(ctx, a, p->dim, grid, st)
                  : write_as<FKV_E4M3, __nv_bfloat16>(ctx, a, p->dim, grid, st);
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
