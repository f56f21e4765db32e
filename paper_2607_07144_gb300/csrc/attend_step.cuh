// What the kernels for a few rows over 8-bit (attend.cu) and 4-bit pages (attend4.cu)
// share: instructions, and the end of a block.
#pragma once

#include "attend.cuh"

namespace fkvd {

constexpr float kPBits = 8.0f;     // the reference's own weight is 2^8: P is at most that over 8-bit pages, 2^15 over 4-bit ones
constexpr int kMaxCluster = 8;     // blocks of a portable cluster

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

__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// The same place in the shared memory of the cluster's block `rank`.
__device__ __forceinline__ uint32_t in_cluster(const float *p, int rank)
{
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
    return a;
}
__device__ __forceinline__ float ld_cluster(const float *p, int rank)
{
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(in_cluster(p, rank)) : "memory");
    return v;
}
__device__ __forceinline__ float4 ld_cluster4(const float *p, int rank)
{
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                 : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
                 : "r"(in_cluster(p, rank))
                 : "memory");
    return v;
}

__device__ __forceinline__ uint32_t transpose8(uint32_t x)
{
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// The end of a block of four warps and 8 NT rows: a row's maxima m, sums l (a lane's
// own keys of rows 2t, 2t + 1) and outputs o (dimensions 2d and 2d + 1 of the lane's
// D / 8; QUADS: of its fours, one in every 32) meet in shared memory, which takes them from `base` on, and the shares of
// a row's keys in their cluster or in the workspace.
template <int D, typename T, int NT, bool QUADS = false>
__device__ __forceinline__ void finish_rows(const AttendArgs &a, const Request &q, uint8_t *base, float (*ml)[2][8 * NT],
                                            const float (&m)[NT][2], const float (&l)[NT][2], const float (&o)[NT][D / 16][4],
                                            int h, int split, int row0, int rows, bool bad)
{
    constexpr int MO = D / 16, R = 8 * NT;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, gid = lane >> 2, t = lane & 3;
    // merge the warps: a row's largest m, then sums and outputs against it
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            float x = l[n][c];
            x += __shfl_xor_sync(~0u, x, 4);
            x += __shfl_xor_sync(~0u, x, 8);
            x += __shfl_xor_sync(~0u, x, 16);
            if (gid == 0) {
                ml[warp][0][8 * n + 2 * t + c] = m[n][c];
                ml[warp][1][8 * n + 2 * t + c] = x;
            }
        }
    if (bad)
        atomicOr(a.status, FKV_ST_RANGE);
    __syncthreads();                   // every ring is read: its memory takes the outputs
    float *mo = reinterpret_cast<float *>(base);
    constexpr int LD = D + 4;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            float *dst = mo + (warp * R + 8 * n + 2 * t + c) * LD + gid * (QUADS ? 4 : D / 8);
#pragma unroll
            for (int d = 0; d < MO; ++d)
                *reinterpret_cast<float2 *>(dst + (QUADS ? 32 * (d >> 1) + 2 * (d & 1) : 2 * d)) = make_float2(o[n][d][c], o[n][d][2 + c]);
        }
    __syncthreads();
    constexpr int TPR = 128 / R, E = D / TPR;      // threads a row, dimensions a thread
    const int row = tid / TPR, c = (tid % TPR) * E;
    const bool live = row0 + row < rows;
    if (!live && !a.cluster)
        return;
    float mt = -INFINITY;
#pragma unroll
    for (int w = 0; w < 4; ++w)
        mt = fmaxf(mt, ml[w][0][row]);
    const float mref = mt == -INFINITY ? 0.0f : mt;
    float lt = 0.0f, f[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const float half = ex2(0.5f * (ml[w][0][row] - mref));
        f[w] = half * half;
        lt += ml[w][1][row] * half * half;
    }
    float inv = lt != 0.0f ? kRef / lt : 0.0f;
    float lse2 = lt != 0.0f ? mref - kPBits + log2f(lt) - kLog2Ref : -INFINITY;
    const int i = live ? static_cast<int>(a.gdiv.div(row0 + row)) : 0;
    const int64_t tok = q.tok0 + i, head = h * a.G + (live ? row0 + row - i * a.G : 0), flat = tok * (a.H * a.G) + head;
    float x[E];
#pragma unroll
    for (int k = 0; k < E; ++k)
        x[k] = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w)
#pragma unroll
        for (int k = 0; k < E; k += 4) {
            const float4 v = *reinterpret_cast<const float4 *>(mo + (w * R + row) * LD + c + k);
            x[k] = fmaf(v.x, f[w], x[k]), x[k + 1] = fmaf(v.y, f[w], x[k + 1]);
            x[k + 2] = fmaf(v.z, f[w], x[k + 2]), x[k + 3] = fmaf(v.w, f[w], x[k + 3]);
        }
    if (a.cluster) {
        // the shares of a row meet in their cluster's shared memory: every block
        // leaves its rows there, and the blocks take every splits-th row
        float *const part = mo + 4 * R * LD, *const part_lse = part + R * D;
#pragma unroll
        for (int k = 0; k < E; k += 4)
            *reinterpret_cast<float4 *>(part + row * D + c + k) = make_float4(x[k] * inv, x[k + 1] * inv, x[k + 2] * inv, x[k + 3] * inv);
        if (c == 0)
            part_lse[row] = lse2;
        cluster_sync();
        const bool mine = live && row % a.splits == split;
        if (mine) {
            float most = -INFINITY, sum = 0.0f, l_s[kMaxCluster];
#pragma unroll
            for (int s = 0; s < kMaxCluster; ++s) {
                l_s[s] = s < a.splits ? ld_cluster(part_lse + row, s) : -INFINITY;
                most = fmaxf(most, l_s[s]);
            }
            const float ref = most == -INFINITY ? 0.0f : most;
#pragma unroll
            for (int k = 0; k < E; ++k)
                x[k] = 0.0f;
#pragma unroll
            for (int s = 0; s < kMaxCluster; ++s) {
                if (s >= a.splits)
                    break;
                const float w = ex2(l_s[s] - ref);
                sum += w;
#pragma unroll
                for (int k = 0; k < E; k += 4) {
                    const float4 v = ld_cluster4(part + row * D + c + k, s);
                    x[k] = fmaf(v.x, w, x[k]), x[k + 1] = fmaf(v.y, w, x[k + 1]);
                    x[k + 2] = fmaf(v.z, w, x[k + 2]), x[k + 3] = fmaf(v.w, w, x[k + 3]);
                }
            }
            inv = sum != 0.0f ? 1.0f / sum : 0.0f;
            lse2 = sum != 0.0f ? ref + log2f(sum) : -INFINITY;
        }
        cluster_sync();                // no block's memory goes before the others have read it
        if (!mine)
            return;
    }
    if (a.splits == 1 || a.cluster) {
        T *dst = static_cast<T *>(a.out) + tok * a.o_tok + head * a.o_head + c;
#pragma unroll
        for (int k = 0; k < E; k += 4) {
            T y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                y[e] = from_float<T>(x[k + e] * inv);
            *reinterpret_cast<uint2 *>(dst + k) = *reinterpret_cast<const uint2 *>(y);
        }
        if (a.lse && c == 0)
            a.lse[flat] = lse2 / kLog2e;
    } else {
        const int64_t at = split * a.T * (a.H * a.G) + flat;
#pragma unroll
        for (int k = 0; k < E; k += 4)
            *reinterpret_cast<float4 *>(a.ws_o + at * D + c + k) =
                make_float4(x[k] * inv, x[k + 1] * inv, x[k + 2] * inv, x[k + 3] * inv);
        if (c == 0)
            a.ws_lse[at] = lse2;
    }
}

}  // namespace fkvd
