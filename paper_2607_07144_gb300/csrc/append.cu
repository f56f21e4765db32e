// Rotary positions on the way into the paged cache (fkv_page_append), and writes of
// 4-bit rows, turned or not (fkv_page_append, fkv_page_write).
//
// A pair (a, b) of a head's dimensions becomes (a c - b s, b c + a s) with the
// position's cosine and sine.  Queries are turned into q_out, keys into codes.  A
// thread holds 16 elements of a head's row in which every pair is whole: for pairs
// i, i + rot / 2 eight from 8 t on and their eight partners, else 16 consecutive
// ones.  Its cosines and sines are the same for every head of the token, so that it
// takes several heads of one token with one look at the tables.
//
// A 4-bit row needs its own extremes alone: middle, step and codes (fkv.h) are
// computed as soon as it is turned, without a look at the page.  8-bit pages share a
// scale among their positions; those blocks follow runs of slots as k_page_write
// does.  One launch does both.
#include "quant.cuh"

using namespace fkvd;

namespace {

constexpr int kAppendThreads = 128;
constexpr float kMost4 = 0x1p102f;           // the largest magnitude of a 4-bit row

struct AppendArgs {
    const void *x[3];                        // queries, keys, values
    int64_t x_tok[3], x_head[3];
    void *q_out;
    int64_t o_tok, o_head;
    uint8_t *pool[2];
    float *scale[2];
    const int64_t *slots;
    const int *pos;                          // or null: nothing is turned
    const float *cos, *sin;
    int64_t T, sb, sh, st, scb, sch, n_slots, n_pos, table_stride;    // n_slots: at most 2^32
    int q_heads, row_heads, heads, per, chunks, run_heads, run_chunks, block, stretch, rot, pairs;
    unsigned row_blocks;                     // blocks that take rows; others take runs of 8-bit pages
    FastDiv by_block, by_heads, by_chunks;
    unsigned *status;
};

// Where a thread's two groups of eight dimensions of a row begin (piece i of D / 16),
// and the rotation of what is there.
struct Groups {
    int d0, d1, f;                           // f: its first cosine, or -1: these are not turned
    __device__ __forceinline__ Groups(const AppendArgs &a, int i)
    {
        const bool on = a.pos && 16 * i < a.rot;
        d0 = on && !a.pairs ? 8 * i : 16 * i;
        d1 = on && !a.pairs ? 8 * i + a.rot / 2 : 16 * i + 8;
        f = on ? 8 * i : -1;
    }
};

// (FIXED: the launch writes nothing of what is read.  Queries may be written in place.)
template <bool FIXED, typename T> __device__ __forceinline__ Raw<T> load_groups(const T *row, const Groups &g)
{
    constexpr int H = sizeof(T) / 2;         // 16-byte words a group
    const uint4 *const p0 = reinterpret_cast<const uint4 *>(row + g.d0), *const p1 = reinterpret_cast<const uint4 *>(row + g.d1);
    Raw<T> r;
#pragma unroll
    for (int i = 0; i < H; ++i) {
        r.v[i] = FIXED ? __ldg(p0 + i) : p0[i];
        r.v[H + i] = FIXED ? __ldg(p1 + i) : p1[i];
    }
    return r;
}

// Eight cosines and sines.
struct Turn {
    float c[8], s[8];
    __device__ __forceinline__ void load(const AppendArgs &a, int64_t p, int f)
    {
        const float4 *cp = reinterpret_cast<const float4 *>(a.cos + p * a.table_stride + f);
        const float4 *sp = reinterpret_cast<const float4 *>(a.sin + p * a.table_stride + f);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float4 u = __ldg(cp + i), v = __ldg(sp + i);
            c[4 * i] = u.x, c[4 * i + 1] = u.y, c[4 * i + 2] = u.z, c[4 * i + 3] = u.w;
            s[4 * i] = v.x, s[4 * i + 1] = v.y, s[4 * i + 2] = v.z, s[4 * i + 3] = v.w;
        }
    }
    __device__ __forceinline__ void pair(float &x, float &y, int e) const
    {
        const float u = __fsub_rn(__fmul_rn(x, c[e]), __fmul_rn(y, s[e])), v = __fadd_rn(__fmul_rn(y, c[e]), __fmul_rn(x, s[e]));
        x = u, y = v;
    }
    __device__ __forceinline__ void apply(float *x, bool pairs) const
    {
        if (pairs) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                pair(x[2 * e], x[2 * e + 1], e);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                pair(x[e], x[8 + e], e);
        }
    }
};

template <typename T> __device__ __forceinline__ void store_groups(T *row, const Groups &g, const float *x)
{
    Raw<T> r;
    store16<T>(reinterpret_cast<T *>(&r), x);
    constexpr int H = sizeof(T) / 2;
#pragma unroll
    for (int i = 0; i < H; ++i) {
        reinterpret_cast<uint4 *>(row + g.d0)[i] = r.v[i];
        reinterpret_cast<uint4 *>(row + g.d1)[i] = r.v[H + i];
    }
}

__device__ __forceinline__ float min_nan(float a, float b)
{
    float y;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}
__device__ __forceinline__ float max_nan(float a, float b)
{
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}

// One row of 4-bit codes by LANES threads of 16 elements each (all of the warp's
// threads take part; `store`: whether the row goes anywhere).
template <int LANES> __device__ __forceinline__ bool put4(float *x, const Groups &g, uint8_t *row, uint32_t *numbers, int lane, bool store)
{
    float lo, hi;
    auto extremes = [&]() {
        lo = x[0], hi = x[0];
#pragma unroll
        for (int e = 1; e < 16; ++e)
            lo = min_nan(lo, x[e]), hi = max_nan(hi, x[e]);
#pragma unroll
        for (int o = 1; o < LANES; o <<= 1) {
            lo = min_nan(lo, __shfl_xor_sync(~0u, lo, o));
            hi = max_nan(hi, __shfl_xor_sync(~0u, hi, o));
        }
    };
    bool nan = false;
    extremes();
    if (__any_sync(~0u, !(lo >= -kMost4 && hi <= kMost4))) {
        // rare: NaN to zero, the rest within the limits
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            nan |= x[e] != x[e];
            x[e] = x[e] != x[e] ? 0.0f : fminf(fmaxf(x[e], -kMost4), kMost4);
        }
        extremes();
    }
    const float mid = __bfloat162float(__float2bfloat16_rn(__fadd_rn(lo * 0.5f, hi * 0.5f)));
    const float reach = fmaxf(__fsub_rn(hi, mid), __fsub_rn(mid, lo));
    const float up = __uint_as_float((__float_as_uint(__fmul_rn(reach, 2.0f / 15.0f)) + 0xffffu) & 0xffff0000u);
    const float step = fmaxf(fmaxf(up, fabsf(mid) * 0x1p-16f), FKV_PAGE_MIN_SCALE);
    const float inv = __frcp_rn(step);
    // Codes lie in -2^-20 .. 15 + 2^-20 before they are rounded.  Adding 1.5 2^23 rounds them;
    // the sums' bits are those of 1.5 2^23 plus the code, and eight of them shifted together
    // hold the eight codes plus a constant.
    constexpr uint32_t bias = 0x4b400000u * 0x11111111u;
    uint32_t w[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        w[k] = 0;
#pragma unroll
        for (int e = 7; e >= 0; --e)
            w[k] = (w[k] << 4) + __float_as_uint(__fadd_rn(__fadd_rn(__fmul_rn(__fsub_rn(x[8 * k + e], mid), inv), 7.5f), 12582912.0f));
        w[k] -= bias;
    }
    if (store) {
        *reinterpret_cast<uint32_t *>(row + g.d0 / 2) = w[0];
        *reinterpret_cast<uint32_t *>(row + g.d1 / 2) = w[1];
        if (lane == 0)
            *numbers = (__float_as_uint(mid) & 0xffff0000u) | __float_as_uint(step) >> 16;
    }
    return nan && store;
}

// Rows by themselves: queries, and 4-bit keys and values.  A warp takes a few tokens
// (D / 16 threads each) and `per` heads of them, several at a time.
template <int D, int FMT, typename T> __device__ __forceinline__ void append_rows(const AppendArgs &a, unsigned task)
{
    constexpr int C = D / 16, R = 32 / C, B = sizeof(T) == 4 ? 2 : 4;       // B heads in flight
    const int lane = threadIdx.x & 31, c = lane % C;
    const unsigned group = a.by_chunks.div(task);
    const int u0 = static_cast<int>(task - group * a.chunks) * a.per, u1 = min(u0 + a.per, a.row_heads);
    const int64_t t = static_cast<int64_t>(group) * R + lane / C;
    if (static_cast<int64_t>(group) * R >= a.T)
        return;
    const Groups g(a, c);
    bool live = t < a.T, range = false, nan = false;
    int64_t slot = -1, p = 0;
    if (live && a.pos) {
        p = a.pos[t];
        range = p >= a.n_pos;
        live = p >= 0 && !range;
    }
    if (FMT == FKV_UINT4 && live) {
        slot = a.slots[t];
        if (slot >= a.n_slots)
            slot = -1, range = true;
    }
    const int64_t blk = slot < 0 ? 0 : a.by_block.div(static_cast<unsigned>(slot));
    const int64_t off = slot - blk * a.block;
    Turn turn;
    if (live && g.f >= 0)
        turn.load(a, p, g.f);
    for (int u = u0; u < u1; u += B) {
        Raw<T> raw[B];
#pragma unroll
        for (int k = 0; k < B; ++k) {
            // queries, then (4-bit pages) keys and values
            const int kind = FMT != FKV_UINT4 || u + k < a.q_heads ? 0 : u + k < a.q_heads + a.heads ? 1 : 2;
            const int h = u + k - (kind == 0 ? 0 : kind == 1 ? a.q_heads : a.q_heads + a.heads);
            if (u + k < u1 && live)
                raw[k] = load_groups<false, T>(static_cast<const T *>(a.x[kind]) + t * a.x_tok[kind] + h * a.x_head[kind], g);
            else
#pragma unroll
                for (int i = 0; i < static_cast<int>(sizeof(T)); ++i)
                    raw[k].v[i] = make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int k = 0; k < B; ++k) {
            if (u + k >= u1)
                break;
            const int kind = FMT != FKV_UINT4 || u + k < a.q_heads ? 0 : u + k < a.q_heads + a.heads ? 1 : 2;
            const int h = u + k - (kind == 0 ? 0 : kind == 1 ? a.q_heads : a.q_heads + a.heads);
            float x[16];
            load16<T>(reinterpret_cast<const T *>(&raw[k]), x);
            if (kind < 2 && g.f >= 0)
                turn.apply(x, a.pairs);
            if (kind == 0) {
                if (live)
                    store_groups<T>(static_cast<T *>(a.q_out) + t * a.o_tok + h * a.o_head, g, x);
            } else if (FMT == FKV_UINT4) {
                uint8_t *const row = a.pool[kind - 1] + blk * a.sb + h * a.sh + off * a.st;
                uint32_t *const numbers = reinterpret_cast<uint32_t *>(a.scale[kind - 1]) + blk * a.scb + h * a.sch + off;
                nan |= put4<C>(x, g, row, numbers, c, slot >= 0);
            }
        }
    }
    if (nan)
        atomicOr(a.status, FKV_ST_CORRUPT);
    if (range)
        atomicOr(a.status, FKV_ST_RANGE);
}

// Runs of slots of 8-bit pages, as k_page_write takes them (paged.cu): GT threads a
// run, some heads, K or V.
template <int D, int FMT, typename T, int GT> __device__ __forceinline__ void append_runs(const AppendArgs &a, unsigned item)
{
    constexpr int C = D / 16, R = GT / C, KEEP = sizeof(T) == 4 ? 2 : 4;        // 16-element pieces a row, rows at a time, kept of them
    __shared__ uint32_t red[GT / 32];
    const int lane = threadIdx.x & 31, tid = GT == 32 ? lane : threadIdx.x, c = tid % C, row0 = tid / C;
    const unsigned both = a.by_heads.div(item);
    const int h0 = static_cast<int>(item - both * a.run_chunks) * a.run_heads, h1 = min(h0 + a.run_heads, a.heads), kv = both & 1;
    const int64_t t0 = static_cast<int64_t>(both >> 1) * a.stretch;
    if (t0 >= a.T)
        return;
    const int64_t t1 = min(t0 + a.stretch, a.T);
    const T *x = static_cast<const T *>(a.x[1 + kv]);
    const int64_t x_tok = a.x_tok[1 + kv], x_head = a.x_head[1 + kv];
    x += h0 * x_head;
    Groups g(a, c);
    if (kv)                                  // values stay as they are
        g.d0 = 16 * c, g.d1 = 16 * c + 8, g.f = -1;
    auto slot_of = [&](int64_t t) {
        const int p = a.pos[t];
        const int64_t s = a.slots[t];
        return p < 0 || p >= a.n_pos ? -1 : s;
    };
    // the thread's elements of a token's row, and what they are turned (twice, for the largest
    // magnitude and the codes: kept turned they would take twice the registers)
    auto raw_of = [&](int64_t t) { return load_groups<true, T>(x + t * x_tok, g); };
    auto turned = [&](const Raw<T> &r, int64_t t, float *v) {
        load16<T>(reinterpret_cast<const T *>(&r), v);
        if (g.f >= 0) {
            Turn turn;
            turn.load(a, a.pos[t], g.f);
            turn.apply(v, a.pairs);
        }
    };
    auto row_of = [&](int64_t t, float *v) { turned(raw_of(t), t, v); };
    auto most_of = [](const float *v, uint32_t m) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
            m = max(m, __float_as_uint(v[e]) & 0x7fffffffu);      // NaN above infinity above numbers
        return m;
    };
    bool nan = false, range = false;
    for (int64_t base = t0; base < t1; base += 32) {
        // a lane a token: which of them begin a run (every warp of a group finds the same)
        const int64_t mine = base + lane;
        int64_t slot_l = -1;
        bool lead = false;
        if (mine < t1) {
            slot_l = slot_of(mine);
            range |= a.pos[mine] >= a.n_pos;
            const int64_t prev = mine > 0 ? slot_of(mine - 1) : -2;
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
            const int most = static_cast<int>(min(static_cast<int64_t>(a.block - off), a.T - t));
            Raw<T> keep[KEEP];
#pragma unroll
            for (int k = 0; k < KEEP; ++k)
                if ((GT > 32 || k == 0) && row0 + k * R < most)
                    keep[k] = raw_of(t + row0 + k * R);
            int len = most;
            for (int i = 0; i < most; i += 32) {
                const unsigned off_run = __ballot_sync(~0u, i + lane < most && slot_of(t + i + lane) != slot + i + lane);
                if (off_run) {
                    len = i + __ffs(off_run) - 1;
                    break;
                }
            }
            // the run's heads, one after the other
            for (int h = h0; h < h1; ++h, x += x_head) {
                float *const sp = a.scale[kv] + blk * a.scb + h * a.sch;
                const float was = off > 0 ? *sp : 0.0f;
                uint8_t *const page = a.pool[kv] + blk * a.sb + h * a.sh;
#pragma unroll
                for (int k = 0; k < KEEP; ++k)
                    if (((GT == 32 && k > 0) || h > h0) && row0 + k * R < len)
                        keep[k] = raw_of(t + row0 + k * R);
                uint32_t amax_u = 0;
#pragma unroll
                for (int k = 0; k < KEEP; ++k)
                    if (row0 + k * R < len) {
                        float v[16];
                        turned(keep[k], t + row0 + k * R, v);
                        amax_u = most_of(v, amax_u);
                    }
                for (int i = row0 + KEEP * R; i < len; i += R) {
                    float v[16];
                    row_of(t + i, v);
                    amax_u = most_of(v, amax_u);
                }
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
                        row_of(t + i, v);
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
                auto put = [&](int row, const uint4 &q) {
                    uint8_t *const p = page + row * a.st;
                    *reinterpret_cast<uint2 *>(p + g.d0) = make_uint2(q.x, q.y);
                    *reinterpret_cast<uint2 *>(p + g.d1) = make_uint2(q.z, q.w);
                };
                if (!odd) {
#pragma unroll
                    for (int k = 0; k < KEEP; ++k)
                        if (row0 + k * R < len) {
                            float v[16];
                            turned(keep[k], t + row0 + k * R, v);
                            put(off + row0 + k * R, codes16_inside<FMT>(v, inv));
                        }
                }
                for (int i = odd ? row0 : row0 + KEEP * R; i < len; i += R) {
                    float v[16];
                    row_of(t + i, v);
                    nan |= drop_nan(v);
                    put(off + i, codes16<FMT>(v, inv));
                }
                __syncwarp();
                if (now != was) {
                    const float ratio = __fmul_rn(was, inv);
                    for (int i = row0; i < off; i += R) {
                        uint4 *p = reinterpret_cast<uint4 *>(page + i * a.st + c * 16);
                        float v[16];
                        values16<FMT>(*p, v);
                        *p = codes16<FMT>(v, ratio);
                    }
                    if (tid == 0)
                        *sp = now;
                }
            }
            x -= (h1 - h0) * x_head;
        }
    }
    if (nan)
        atomicOr(a.status, FKV_ST_CORRUPT);
    if (range)
        atomicOr(a.status, FKV_ST_RANGE);
}

// Bytes bound long calls, and a few blocks an SM more or less what is in flight of them: 9
// prompts of 1,000 to 8,192 tokens (32 query and 8 KV heads of 128, bf16) into 4-bit pages
// 193 us, 5.6 TB/s, with six blocks an SM (80 registers, 24 to 48 bytes a thread spilled), 216
// without the limit, 252 with eight (64 registers, more spilled); into e4m3 pages 207 us with five (with one head a run 242, 277 with six blocks, 335 with turned
// rows kept in fp32).
template <int D, int FMT, typename T, int GT> __global__ void __launch_bounds__(kAppendThreads, FMT == FKV_UINT4 ? 6 : 5) k_page_append(const AppendArgs a)
{
    if constexpr (FMT == FKV_UINT4) {
        append_rows<D, FMT, T>(a, blockIdx.x * (kAppendThreads / 32) + (threadIdx.x >> 5));
    } else {
        // the runs, whose chains are longer, first (238 us against 242)
        const unsigned runs = gridDim.x - a.row_blocks;
        if (blockIdx.x >= runs)
            append_rows<D, FMT, T>(a, (blockIdx.x - runs) * (kAppendThreads / 32) + (threadIdx.x >> 5));
        else
            append_runs<D, FMT, T, GT>(a, GT == 32 ? blockIdx.x * (kAppendThreads / 32) + (threadIdx.x >> 5) : blockIdx.x);
    }
}

// Heads a warp takes, with one look at the tables: as many as leave every SM 16 warps (with
// 64, small heads looked at them twice as often: 23 us against 19 for 13 GPT-2-shaped prompts).
int append_heads(const fkv_ctx *ctx, int64_t groups, int heads)
{
    const int64_t tasks = groups * heads, most = static_cast<int64_t>(ctx->sms) * 16;
    const int64_t per = tasks / most;
    return static_cast<int>(per < 1 ? 1 : per > 16 ? 16 : per);
}

// Whether a run is a warp's: a step's, and where that makes four rows a lane at most: a
// block's other threads would have none (13 GPT-2-shaped prompts, pages of 16: 31 us against 52).
bool warp_runs(const AppendArgs &a, int dim) { return a.stretch == 1 || a.block * (dim / 16) <= 32 * 4; }

template <int D, int FMT, typename T> cudaError_t append_as(const AppendArgs &a, cudaStream_t st)
{
    if (FMT == FKV_UINT4) {
        k_page_append<D, FMT, T, 32><<<a.row_blocks, kAppendThreads, 0, st>>>(a);
        return cudaGetLastError();
    }
    const int64_t items = (a.T + a.stretch - 1) / a.stretch * 2 * a.run_chunks;
    if (warp_runs(a, D))
        k_page_append<D, FMT, T, 32><<<a.row_blocks + static_cast<unsigned>((items + 3) / 4), kAppendThreads, 0, st>>>(a);
    else
        k_page_append<D, FMT, T, FMT == FKV_UINT4 ? 32 : kAppendThreads>
            <<<a.row_blocks + static_cast<unsigned>(items), kAppendThreads, 0, st>>>(a);
    return cudaGetLastError();
}

template <int FMT, typename T> cudaError_t append_dim(const AppendArgs &a, int dim, cudaStream_t st)
{
    return dim == 64 ? append_as<64, FMT, T>(a, st) : append_as<128, FMT, T>(a, st);
}

template <int FMT> cudaError_t append_type(const AppendArgs &a, int dim, int dtype, cudaStream_t st)
{
    return dtype == FKV_F32   ? append_dim<FMT, float>(a, dim, st)
           : dtype == FKV_F16 ? append_dim<FMT, __half>(a, dim, st)
                              : append_dim<FMT, __nv_bfloat16>(a, dim, st);
}

}  // namespace

// rot 0: a write without a rotation (4-bit pages).
cudaError_t launch_page_append(const fkv_ctx *ctx, const fkv_pages *p, const fkv_rotary &r, cudaStream_t st)
{
    AppendArgs a;
    const void *x[3] = {r.q, r.k, r.v};
    const int64_t tok[3] = {r.q_stride_tok, r.k_stride_tok, r.v_stride_tok};
    const int64_t head[3] = {r.q_stride_head, r.k_stride_head, r.v_stride_head};
    for (int i = 0; i < 3; ++i)
        a.x[i] = x[i], a.x_tok[i] = tok[i], a.x_head[i] = head[i];
    a.q_out = r.q_out, a.o_tok = r.out_stride_tok, a.o_head = r.out_stride_head;
    a.pool[0] = static_cast<uint8_t *>(p->k), a.pool[1] = static_cast<uint8_t *>(p->v);
    a.scale[0] = p->k_scale, a.scale[1] = p->v_scale;
    a.slots = r.slots, a.pos = r.rot ? r.pos : nullptr, a.cos = r.cos, a.sin = r.sin;
    a.T = r.n_tok, a.sb = p->stride_block, a.sh = p->stride_head, a.st = p->stride_pos;
    a.scb = p->scale_stride_block, a.sch = p->scale_stride_head;
    a.n_slots = p->n_blocks * p->block, a.n_pos = r.n_pos, a.table_stride = r.table_stride;
    a.q_heads = r.q ? r.n_q_heads : 0, a.heads = p->n_heads, a.block = p->block, a.rot = r.rot, a.pairs = r.interleaved;
    a.row_heads = a.q_heads + (p->format == FKV_UINT4 ? 2 * p->n_heads : 0);
    a.status = ctx->d_status;
    // the rule of k_page_write (paged.cu): a warp a token, or a block a page's worth
    a.stretch = a.T * p->n_heads * 2 <= static_cast<int64_t>(ctx->sms) * 64 ? 1 : p->block;
    const int tokens = 32 / (p->dim / 16);
    const int64_t groups = (a.T + tokens - 1) / tokens;
    a.per = append_heads(ctx, groups, a.row_heads);
    a.chunks = (a.row_heads + a.per - 1) / a.per;
    a.row_blocks = static_cast<unsigned>((groups * a.chunks + kAppendThreads / 32 - 1) / (kAppendThreads / 32));
    // Heads a run is looked up for: up to four, in equal parts, while an SM keeps 64 warps or 16
    // blocks of runs (60 GPT-2-shaped prompts 86 us, 101 with one, 111 with twelve; Llama-shaped
    // ones 207, 242, 199 with eight).
    const int64_t runs = (a.T + a.stretch - 1) / a.stretch * 2, room = static_cast<int64_t>(ctx->sms) * (warp_runs(a, p->dim) ? 64 : 16);
    const int64_t want = a.stretch == 1 ? 1 : runs * a.heads / room;
    const int at_most = static_cast<int>(want < 1 ? 1 : want > 4 ? 4 : want);
    a.run_chunks = (a.heads + at_most - 1) / at_most;
    a.run_heads = (a.heads + a.run_chunks - 1) / a.run_chunks;
    a.by_block = FastDiv::make(static_cast<unsigned>(p->block)), a.by_heads = FastDiv::make(static_cast<unsigned>(a.run_chunks));
    a.by_chunks = FastDiv::make(static_cast<unsigned>(a.chunks ? a.chunks : 1));
    switch (p->format) {
    case FKV_E4M3:
        return append_type<FKV_E4M3>(a, p->dim, r.dtype, st);
    case FKV_INT8:
        return append_type<FKV_INT8>(a, p->dim, r.dtype, st);
    default:
        return append_type<FKV_UINT4>(a, p->dim, r.dtype, st);
    }
}

int64_t page_append_blocks(const fkv_pages *p, const fkv_rotary &r)
{
    const int64_t heads = (r.q ? r.n_q_heads : 0) + (p->format == FKV_UINT4 ? 2 * p->n_heads : 0);
    return (r.n_tok + 3) / 4 * heads + (p->format == FKV_UINT4 ? 0 : (r.n_tok / p->block + 1) * 2 * p->n_heads);
}
