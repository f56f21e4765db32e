// Attention over the paged 8-bit K/V cache (fkv_page_attend).
//
// For a query row (token i of request r, query head u of KV head h) at position
// p = kv_len - n_new + i, with c the codes of a page and ks, vs its scales,
//     x_j = f(scale ks q.c_j) + slope (j - p),   f(s) = cap tanh(s / cap) or s
//     o   = sum_j exp(x_j) vs c'_j / sum_j exp(x_j)   over the visible j.
// Codes are exact in fp16, and so is a query row brought to [2^14, 2^15) by a
// power of two (fp16 queries as they are), but for a bf16 row's elements below
// 2^-31 of its largest, which fp16's subnormals round to 2^-39 of that: the products
// are exact and summed in fp32 on the tensor cores, and the scale of a page
// multiplies afterwards, once for each score.  The value scale goes into the
// softmax instead: with
//     y_j = x_j log2 e + log2 vs,    P_j = 2^(y_j - m + 8),   m = max y_j
// the second product is sum P_j c'_j with P rounded to fp16 (relative 2^-11, an
// eighth of a bf16 result's own rounding; P spans 2^8 .. 2^-24, so nothing above
// 2^-32 of the largest weight is lost), and the sum of the weights is
// sum P_j / vs, from the unrounded P_j, in fp32 (share_of).  So pages of any
// scales mix in one accumulator without a rounding of V.
#include <algorithm>

#include "attend_step.cuh"

using namespace fkvd;

namespace {

// ------------------------------------------------------------------ steps --
// Up to 8 NT rows (the query heads of a KV head, times the new tokens) against a
// share of the keys: bound by reading the pages.  A warp owns every fourth
// group of 32 keys, loads it by TMA into a ring of its own and keeps its own
// running maximum, sum and output, so nothing but the last merge joins the
// warps.  Keys are the rows of the first product and dimensions those of the
// second, so the pages' codes are both times the operand of 16 rows and the few
// query rows the one of 8 columns:
//     S[key][row] = K Q^T,    O^T[dim][row] = V^T P^T,
// with a transpose of 8 x 8 weights between them.  Codes become fragments in
// registers: the contraction may run over the dimensions in any order, so a lane
// takes 16 consecutive bytes of a key as four steps' operands, and 16 bytes of a
// value row as 16 rows of the result.  mma.sync, as these shapes are a sixteenth
// of what tcgen05 multiplies at least; its rate leaves the bytes the bound.
// 8 heads of 128, 4 rows each: 64 sequences of 16-32k positions, e4m3, 497 us, 6.6
// TB/s; one of 131k, int8 with a cap, 52 us, 5.2 TB/s (the codes' conversion).  Up
// to 28 rows, 24 sequences, a window of 4,096, a bias: 88 us, 2.3 TB/s (the chain of a
// warp's iteration, and two tiles of rows that read the keys each).
template <int D, int NT> struct StepShape {
    static constexpr int stages = D == 128 ? 2 : 4, ring = 4 * stages * 64 * D;
    // more than 8 rows: the query operands, [column tile][step][lane]
    static constexpr int q = NT > 1 ? NT * (D / 16) * 256 : 0, ml = 4 * 2 * 8 * NT * 4;
    static constexpr int smem = ring + q + ml + 1024;
};

template <int D, int FMT, typename T, int NT>
__global__ void __launch_bounds__(128, 3)
    k_attend_step(const AttendArgs a, const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv)
{
    constexpr int ST = StepShape<D, NT>::stages, NS = D / 64, UNIT = 16 * D, STAGE = 4 * UNIT, MO = D / 16, R = 8 * NT;
    extern __shared__ uint8_t raw[];
    __shared__ __align__(8) uint64_t bars[4 * ST];
    __shared__ Seen rows_see[4];                 // a warp's own: registers are short
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, gid = lane >> 2, t = lane & 3;
    const uint32_t sbase = (smem_u32(raw) + 1023) & ~1023u;
    uint8_t *const base = raw + (sbase - smem_u32(raw));
    uint2 *const q_s = reinterpret_cast<uint2 *>(base + StepShape<D, NT>::ring);
    typedef float RowPair[2][R];                 // a warp's maxima and sums
    RowPair *const ml = reinterpret_cast<RowPair *>(base + StepShape<D, NT>::ring + StepShape<D, NT>::q);

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
    // the last tile may end before this warp's keys
    const int n_it = max(0, i1 - i0) - (i1 > i0 && tiles.at(i1 - 1) * kTile + warp * 32 >= tiles.lim);
    // A bias by distance grows along the keys, and the maximum with it, so that the
    // outputs are scaled at every iteration: biased scores are walked from the last
    // tile back.
    const bool back = a.slopes != nullptr;
    auto tile_at = [&](int it) { return tiles.at(i0 + (back ? n_it - 1 - it : it)); };

    const uint32_t ring = sbase + warp * ST * STAGE, bar0 = smem_u32(bars) + warp * ST * 8;
    if (lane == 0) {
        rows_see[warp] = tiles.seen;
        for (int s = 0; s < ST; ++s)
            mbar_init(bar0 + 8 * s, 1);
        fence_mbar_init();
    }
    __syncwarp();

    // A lane looks up one of the 32 units (16 keys) of 16 iterations, if any row sees
    // one of its keys: its page and what its scales give the scores.  Page ids are
    // asked for a batch of iterations before the scales, and these a batch before
    // their use, so that no warp waits for one to ask for the other.
    struct Unit {
        int id;
        float ks, vs;
        unsigned all;                  // which of the 32 units are looked at
    };
    const float mul0 = score_multiplier(a, a.scale);
    bool bad = false;
    auto key_of = [&](int batch) { return tile_at(batch * 16 + (lane >> 1)) * kTile + warp * 32 + (lane & 1) * 16; };
    auto on = [&](int batch) { return batch * 16 + (lane >> 1) < n_it && rows_see[warp].of(key_of(batch)); };
    auto ask = [&](int batch) { return on(batch) ? a.table[r * a.table_stride + a.div.div(key_of(batch))] : 0; };
    auto ask_scales = [&](int batch, int id) {
        const bool mine = on(batch);
        Unit u = {0, 0.0f, 1.0f, __ballot_sync(~0u, mine)};
        if (mine) {
            if (id < 0 || id >= a.n_blocks)
                bad = true;
            else
                u.id = id;
            u.ks = a.ks[u.id * a.scb + h * a.sch], u.vs = a.vs[u.id * a.scb + h * a.sch];
        }
        return u;
    };
    int nid = ask(0), nnid = ask(1);
    Unit cur = ask_scales(0, nid), nxt = ask_scales(1, nnid);
    nid = ask(2);
    auto first_key = [&](int it) { return tile_at(it) * kTile + warp * 32; };
    auto issue = [&](int it, int batch) {
        const int from = (it & 15) * 2 + (lane & 1);
        const bool now = (it >> 4) == batch;
        const unsigned units = (now ? cur.all : nxt.all) >> ((it & 15) * 2) & 3;
        const int id = __shfl_sync(~0u, now ? cur.id : nxt.id, from);
        const int key = first_key(it) + (lane & 1) * 16, off = key - static_cast<int>(a.div.div(key)) * a.block;
        const uint32_t bar = bar0 + 8 * (it % ST), dst = ring + (it % ST) * STAGE;
        // (without any the arrival alone completes the phase)
        if (lane == 0)
            mbar_arrive_expect_tx(bar, __popc(units) * 2 * UNIT);
        __syncwarp();
        // lanes 0 .. 3: units 0 and 1 of K, then of V
        if (lane < 4 && (units >> (lane & 1) & 1))
            tma_load_4d(dst + lane * UNIT, lane < 2 ? &mk : &mv, 0, off, h, id, bar);
        __syncwarp();
    };
    for (int it = 0; it < min(ST - 1, n_it); ++it)
        issue(it, 0);

    // the query rows as fp16 operands: lane t's steps take 16 consecutive
    // dimensions (two such pieces for D = 128) of row gid
    uint32_t qf[NT > 1 ? 1 : NS * 4][2];
    float rowmul[NT][2], slope[NT][2];
    int prow[NT][2], hi[NT][2], from[NT][2], pre[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int row = row0 + 8 * n + gid;
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
        // bf16 rows: 2^(14 - exponent), so that fp16 holds them (see above)
        float up = 1.0f, down = 1.0f;
        if (!std::is_same<T, __half>::value) {
            amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, 1));
            amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, 2));
            const int e = max(static_cast<int>(__float_as_uint(amax) >> 23) - 127, -100);
            up = __uint_as_float(static_cast<uint32_t>(127 + 14 - e) << 23);
            down = __uint_as_float(static_cast<uint32_t>(127 - 14 + e) << 23);
        }
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
                const uint32_t f0 = pack_half(x[s][4 * kk] * up, x[s][4 * kk + 1] * up);
                const uint32_t f1 = pack_half(x[s][4 * kk + 2] * up, x[s][4 * kk + 3] * up);
                if (NT > 1) {
                    if (warp == n % 4)
                        q_s[(n * NS * 4 + s * 4 + kk) * 32 + lane] = make_uint2(f0, f1);
                } else {
                    qf[s * 4 + kk][0] = f0, qf[s * 4 + kk][1] = f1;
                }
            }
        // a lane's scores are of rows 2t and 2t + 1
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            rowmul[n][c] = __shfl_sync(~0u, down, (2 * t + c) * 4);
            const int rw = row0 + 8 * n + 2 * t + c;
            const bool on = rw < rows;
            const int ii = on ? static_cast<int>(a.gdiv.div(rw)) : 0;
            prow[n][c] = q.p0 + ii;
            slope[n][c] = a.slopes && on ? a.slopes[h * a.G + rw - ii * a.G] * kLog2e : 0.0f;
            const RowMask m(a, q, prow[n][c], on);
            hi[n][c] = m.hi, from[n][c] = m.from, pre[n][c] = m.pre;
        }
    }

    if (NT > 1)
        __syncthreads();

    float o[NT][MO][4];
    float m[NT][2], l[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int d = 0; d < MO; ++d)
            o[n][d][0] = o[n][d][1] = o[n][d][2] = o[n][d][3] = 0.0f;
        m[n][0] = m[n][1] = -INFINITY;
        l[n][0] = l[n][1] = 0.0f;
    }

    // the scores' multiplier, the logarithm of V's scale, and what a weight counts
    float cur_mul, cur_lvs, cur_ivs;
    auto finish = [&]() {
        const float vs = value_scale(cur.vs);
        cur_mul = cur.ks * mul0, cur_lvs = lg2(vs), cur_ivs = share_of(vs);
    };
    finish();
    int batch = 0;
    for (int it = 0; it < n_it; ++it) {
        if ((it >> 4) != batch) {
            batch = it >> 4;
            cur = nxt;
            finish();
            nxt = ask_scales(batch + 1, nid);
            nid = ask(batch + 2);
        }
        if (it + ST - 1 < n_it)
            issue(it + ST - 1, batch);
        const int key = first_key(it);
        const unsigned units = cur.all >> ((it & 15) * 2) & 3;
        // (a lane that gives up takes its warp along: the others would meet it nowhere)
        if (!__all_sync(~0u, mbar_wait(bar0 + 8 * (it % ST), (it / ST) & 1, a.status))) {
            // give the loads in flight a while to land before the memory is used again
            for (int k = it + 1; k < min(n_it, it + ST); ++k)
                mbar_wait(bar0 + 8 * (k % ST), (k / ST) & 1, a.status, 2000000);
            __syncwarp();
            break;
        }
        if (units == 0)
            continue;                  // keys between the first ones and the window
        const uint32_t kt = ring + (it % ST) * STAGE, vt = kt + 2 * UNIT;

        float sc[2][NT][4];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int n = 0; n < NT; ++n)
                sc[u][n][0] = sc[u][n][1] = sc[u][n][2] = sc[u][n][3] = 0.0f;
        // both units' keys gid and gid + 8; a unit that was not loaded gives
        // products of any bytes, which no row sees
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            const int c = NS * t + s;
            uint4 w[2][2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int kr = 16 * u + gid;
                const uint32_t at = D == 128 ? kt + kr * 128 + ((c ^ (kr & 7)) << 4) : kt + kr * 64 + ((c ^ ((kr >> 1) & 3)) << 4);
                w[u][0] = lds128(at), w[u][1] = lds128(at + 8 * D);
            }
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
                uint32_t f[2][4];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    codes4_half<FMT>(reinterpret_cast<const uint32_t *>(&w[u][0])[kk], f[u][0], f[u][2]);
                    codes4_half<FMT>(reinterpret_cast<const uint32_t *>(&w[u][1])[kk], f[u][1], f[u][3]);
                }
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    uint2 qv;
                    if (NT > 1)
                        qv = q_s[(n * NS * 4 + s * 4 + kk) * 32 + lane];
                    else
                        qv = make_uint2(qf[s * 4 + kk][0], qf[s * 4 + kk][1]);
                    mma16816(sc[0][n], f[0], qv.x, qv.y);
                    mma16816(sc[1][n], f[1], qv.x, qv.y);
                }
            }
        }

        // scores in base 2 with the value scales' logarithms
        float mx[NT][2], ivs[2];
#pragma unroll
        for (int n = 0; n < NT; ++n)
            mx[n][0] = mx[n][1] = -INFINITY;
        const bool full = all_see(a, q, pa, pb, key, key + 32);
        float bias[NT][2];
        if (a.slopes) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int c = 0; c < 2; ++c)
                    bias[n][c] = slope[n][c] * static_cast<float>(key + gid - prow[n][c]);
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int at = (it & 15) * 2 + u;
            const float mul = __shfl_sync(~0u, cur_mul, at), lvs = __shfl_sync(~0u, cur_lvs, at);
            ivs[u] = __shfl_sync(~0u, cur_ivs, at);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                float x[4];
                if (a.softcap > 0.0f && plain_cap(a)) {
                    const float cap = a.cap2;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float z = ex2(sc[u][n][e] * (mul * rowmul[n][e & 1]));
                        x[e] = fmaf(-2.0f * cap, __fdividef(1.0f, 1.0f + z), cap + lvs);
                    }
                } else if (a.softcap > 0.0f) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        x[e] = capped(a, sc[u][n][e] * (mul * rowmul[n][e & 1])) + lvs;
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        x[e] = fmaf(sc[u][n][e], mul * rowmul[n][e & 1], lvs);
                }
                if (a.slopes) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        x[e] = fmaf(slope[n][e & 1], static_cast<float>(16 * u + 8 * (e >> 1)), x[e] + bias[n][e & 1]);
                }
                if (!full) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int j = key + 16 * u + gid + 8 * (e >> 1), c = e & 1;
                        const bool see = (j < hi[n][c] && (j >= from[n][c] || j < a.sinks)) || j < pre[n][c];
                        x[e] = see ? x[e] : -INFINITY;
                    }
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    sc[u][n][e] = x[e];
                    mx[n][e & 1] = fmaxf(mx[n][e & 1], x[e]);
                }
            }
        }
        bool grown = false;
        float mref[NT][2], by[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                float x = mx[n][c];
                x = fmaxf(x, __shfl_xor_sync(~0u, x, 4));
                x = fmaxf(x, __shfl_xor_sync(~0u, x, 8));
                x = fmaxf(x, __shfl_xor_sync(~0u, x, 16));
                const float mn = fmaxf(m[n][c], x);
                grown |= mn != m[n][c];
                mref[n][c] = (mn == -INFINITY ? 0.0f : mn) - kPBits;
                by[n][c] = m[n][c] - kPBits - mref[n][c];
                m[n][c] = mn;
            }
        if (__any_sync(~0u, grown)) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                // a sum is scaled in two halves: counted up to 2^80 a weight (share_of), it
                // outlasts factors below float32's least
                const float h0 = ex2(0.5f * by[n][0]), h1 = ex2(0.5f * by[n][1]), f0 = h0 * h0, f1 = h1 * h1;
                l[n][0] = l[n][0] * h0 * h0, l[n][1] = l[n][1] * h1 * h1;
#pragma unroll
                for (int d = 0; d < MO; ++d) {
                    o[n][d][0] *= f0, o[n][d][1] *= f1;
                    o[n][d][2] *= f0, o[n][d][3] *= f1;
                }
            }
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            if (!(units >> u & 1))
                continue;
            uint32_t pf[NT][2];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                float p[4];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    p[e] = ex2(sc[u][n][e] - mref[n][e & 1]);
                l[n][0] = fmaf(p[0] + p[2], ivs[u], l[n][0]);
                l[n][1] = fmaf(p[1] + p[3], ivs[u], l[n][1]);
                pf[n][0] = transpose8(pack_half(p[0], p[1]));
                pf[n][1] = transpose8(pack_half(p[2], p[3]));
            }
            // value rows 2t, 2t + 1, 2t + 8, 2t + 9 of the unit, D / 8 dimensions
            // each; those that a row does not see hold any bytes, and a weight of zero
            // does not undo a NaN code
            uint32_t w[4][D / 32];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int row = 16 * u + 2 * t + (x & 1) + 8 * (x >> 1);
                if (D == 128) {
                    const uint4 v = lds128(vt + row * 128 + ((gid ^ (row & 7)) << 4));
                    w[x][0] = v.x, w[x][1] = v.y;
                    w[x][D / 32 - 2] = v.z, w[x][D / 32 - 1] = v.w;
                } else {
                    const uint2 v = lds64(vt + row * 64 + ((((gid >> 1) ^ ((row >> 1) & 3)) << 4) | (gid & 1) << 3));
                    w[x][0] = v.x, w[x][1] = v.y;
                }
            }
            if (FMT == FKV_E4M3 && !full) {
#pragma unroll
                for (int x = 0; x < 4; ++x)
#pragma unroll
                    for (int k = 0; k < D / 32; ++k)
                        w[x][k] = without_nan(w[x][k]);
            }
#pragma unroll
            for (int k = 0; k < D / 32; ++k)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    // rows gid and gid + 8 of the tile: dimensions 4k + 2e and the next
                    const int sel = e ? 0x7362 : 0x5140;
                    uint32_t f[4];
                    codes4_half<FMT>(__byte_perm(w[0][k], w[1][k], sel), f[0], f[1]);
                    codes4_half<FMT>(__byte_perm(w[2][k], w[3][k], sel), f[2], f[3]);
#pragma unroll
                    for (int n = 0; n < NT; ++n)
                        mma16816(o[n][2 * k + e], f, pf[n][0], pf[n][1]);
                }
        }
        __syncwarp();                  // the stage is free: the next issue may overwrite it
    }

    finish_rows<D, T, NT>(a, q, base, ml, m, l, o, h, split, row0, rows, bad);
}

// --------------------------------------------------------------- combine --
// A block per query row: the splits' outputs weighted by 2^(lse - largest).
// Its four warps take every fourth split (two at a time for 64 dimensions), so
// that the loads of a row are in flight together: latency bounds the call (some
// 3 us behind the shares' kernel, whose end its launch overlaps).
constexpr int kMaxSplits = 64;

template <int D, typename T> __global__ void __launch_bounds__(128) k_attend_combine(const AttendArgs a)
{
    constexpr int L = D / 4, P = 128 / L;          // lanes a row of 4 dimensions each, splits at a time
    __shared__ float w_s[kMaxSplits];
    __shared__ float4 part[P][L];
    const int tid = threadIdx.x, lane = tid & 31, g = tid / L, c = tid % L;
    const int64_t Hq = a.H * a.G, row = blockIdx.x, tok = row / Hq, head = row - tok * Hq;
    // rows behind the last request's are no one's, and those of a request that
    // was skipped have no partial results: both are left as they are
    int lo = 0, hi = a.n_req;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.cu[mid] <= tok)
            lo = mid;
        else
            hi = mid;
    }
    Request q;
    bool mine = q.load(a, lo) && tok >= q.tok0 && tok < q.tok0 + q.nq;
    if (!mine) {
        // requests whose numbers do not hold together may have led the search astray
        bool any = false;
        for (int r = tid; r < a.n_req; r += 128)
            any |= q.load(a, r) && tok >= q.tok0 && tok < q.tok0 + q.nq;
        mine = __syncthreads_or(any);
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");     // the partial results are written
    if (!mine)
        return;
    if (tid < kMaxSplits)
        w_s[tid] = tid < a.splits ? a.ws_lse[tid * a.T * Hq + row] : -INFINITY;
    __syncthreads();
    float mx = fmaxf(w_s[lane], w_s[lane + 32]);
#pragma unroll
    for (int o = 16; o; o >>= 1)
        mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, o));
    const float mref = mx == -INFINITY ? 0.0f : mx;
    float sum = ex2(w_s[lane] - mref) + ex2(w_s[lane + 32] - mref);
#pragma unroll
    for (int o = 16; o; o >>= 1)
        sum += __shfl_xor_sync(~0u, sum, o);
    float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
    for (int s = g; s < a.splits; s += P) {
        const float w = ex2(w_s[s] - mref);
        const float4 v = *reinterpret_cast<const float4 *>(a.ws_o + (s * a.T * Hq + row) * D + 4 * c);
        // a split without a visible key has weight zero (its output is zeros)
        x.x = fmaf(w, v.x, x.x), x.y = fmaf(w, v.y, x.y), x.z = fmaf(w, v.z, x.z), x.w = fmaf(w, v.w, x.w);
    }
    part[g][c] = x;
    __syncthreads();
    if (g != 0)
        return;
#pragma unroll
    for (int k = 1; k < P; ++k) {
        const float4 v = part[k][c];
        x.x += v.x, x.y += v.y, x.z += v.z, x.w += v.w;
    }
    const float inv = sum != 0.0f ? 1.0f / sum : 0.0f;
    const T y[4] = {from_float<T>(x.x * inv), from_float<T>(x.y * inv), from_float<T>(x.z * inv), from_float<T>(x.w * inv)};
    *reinterpret_cast<uint2 *>(static_cast<T *>(a.out) + tok * a.o_tok + head * a.o_head + 4 * c) =
        *reinterpret_cast<const uint2 *>(y);
    if (a.lse && c == 0)
        a.lse[row] = sum != 0.0f ? (mref + log2f(sum)) / kLog2e : -INFINITY;
}

// ------------------------------------------------------------------ launch --
// A window that holds every position is none.
int window_of(const fkv_attend &c) { return c.window >= FKV_PAGE_MAX_LEN ? 0 : static_cast<int>(c.window); }

template <int D, int FMT, typename T, int NT>
cudaError_t step_rows(const fkv_ctx *ctx, const AttendArgs &a, const CUtensorMap &mk, const CUtensorMap &mv, cudaStream_t st)
{
    const void *fn = reinterpret_cast<const void *>(k_attend_step<D, FMT, T, NT>);
    const cudaError_t e = kernel_use(ctx, fn, 128, StepShape<D, NT>::smem, nullptr);
    if (e != cudaSuccess)
        return e;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = a.cluster ? a.splits : 1, at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(a.n_req * a.row_tiles * a.splits), a.H), cfg.blockDim = dim3(128);
    cfg.dynamicSmemBytes = StepShape<D, NT>::smem, cfg.stream = st;
    cfg.attrs = &at, cfg.numAttrs = a.cluster ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, k_attend_step<D, FMT, T, NT>, a, mk, mv);
}

template <int D, int FMT, typename T>
cudaError_t step_as(const fkv_ctx *ctx, const AttendArgs &a, int nt, const CUtensorMap &mk, const CUtensorMap &mv,
                    cudaStream_t st)
{
    const cudaError_t e = nt == 0   ? launch_attend_prompt(ctx, a, D, FMT, std::is_same<T, __half>::value ? FKV_F16 : FKV_BF16, st)
                          : nt == 1 ? step_rows<D, FMT, T, 1>(ctx, a, mk, mv, st)
                                    : step_rows<D, FMT, T, 2>(ctx, a, mk, mv, st);
    if (e != cudaSuccess || a.splits == 1 || a.cluster)
        return e;
    return launch_after(k_attend_combine<D, T>, static_cast<unsigned>(a.T * a.H * a.G), 128, 0, st, a);
}

template <int D, typename T>
cudaError_t step4_as(const fkv_ctx *ctx, const AttendArgs &a, int nt, const CUtensorMap &mk, const CUtensorMap &mv, cudaStream_t st)
{
    const int dtype = std::is_same<T, __half>::value ? FKV_F16 : FKV_BF16;
    const cudaError_t e = nt == 0 ? launch_attend_prompt4(ctx, a, D, dtype, st) : launch_attend_step4(ctx, a, D, dtype, nt, mk, mv, st);
    if (e != cudaSuccess || a.splits == 1 || a.cluster)
        return e;
    return launch_after(k_attend_combine<D, T>, static_cast<unsigned>(a.T * a.H * a.G), 128, 0, st, a);
}

template <int D, int FMT>
cudaError_t step_dt(const fkv_ctx *ctx, const AttendArgs &a, int dtype, int nt, const CUtensorMap &mk, const CUtensorMap &mv,
                    cudaStream_t st)
{
    return dtype == FKV_F16 ? step_as<D, FMT, __half>(ctx, a, nt, mk, mv, st)
                            : step_as<D, FMT, __nv_bfloat16>(ctx, a, nt, mk, mv, st);
}

}  // namespace

// Which kernel serves the call, and how many shares the keys are split into.
// Up to 32 rows a KV head (in tiles of nt = 1 or 2 columns of 8) go to the step
// kernel, more to the tensor-memory one (nt = 0): for 24 sequences of 3-16k
// positions and 8 heads of 128 in 8-bit pages, 63 rows take 384 us against 236; 28 rows 265
// against 224 and 274 against 263 with a bias, but 84 against 110 with a window of
// 4,096 and 283 against 364 with a cap.  (4-bit pages: 28 rows 205 us, 32 rows 217,
// 36 by the tensor-memory kernel 324.)  A block's time is its keys plus a fixed
// part (its launch, the first loads' latency and its end: about that of 384 keys);
// the blocks run in waves of `slots`.  The split with the least waves x time wins.
// Up to eight shares of the step kernel are joined in their cluster (about 100
// keys' time) if all blocks run at once: where blocks queue,
// those of a cluster hold their places until its last one is done (64 ragged
// sequences of 16-32k positions: 561 us, and 499 with the shares joined by
// another launch, which costs 512 keys' time and 8 a share).
fkv_attend_plan page_attend_plan(const fkv_ctx *ctx, const fkv_attend &c)
{
    fkv_attend_plan p;
    const int H = c.pages->n_heads, G = c.n_q_heads / H, window = window_of(c);
    const int64_t most = c.max_new * G;
    p.nt = most <= 8 ? 1 : most <= 32 ? 2 : 0;
    const int per = p.nt ? 8 * p.nt : prompt_rows();
    p.row_tiles = static_cast<int>((most + per - 1) / per);
    const int64_t blocks = c.n_req * H * p.row_tiles, slots = ctx->sms * (p.nt == 0 ? 1 : c.pages->format == FKV_UINT4 ? step4_blocks(p.nt) : 3);
    // Of 4-bit pages, the blocks that will have rows, as far as the number of tokens tells:
    // others end at once, and no wave has to be saved for them (24 requests of 2 to 7 tokens,
    // 4 query heads each: 66 us, 83 with all their second tiles counted).  n_req / 3 is what
    // those requests' last tiles lack of full ones; it has been measured there alone, and a
    // wrong guess costs a share more or less.
    int64_t busy = blocks;
    if (c.pages->format == FKV_UINT4) {
        const int64_t tiles = std::max(std::min(c.n_req, c.n_tok), (c.n_tok * G + per - 1) / per + c.n_req / 3);
        busy = H * std::min(tiles, c.n_req * p.row_tiles);
    }
    // all that a block of rows may look at: with a window, that and the sinks (whose
    // tiles end apart); a prefix may be of any length
    int64_t span = c.max_len;
    const int64_t seen = c.window + c.max_new + 2 * kTile + (c.sinks > 0 ? c.sinks + kTile : 0);
    if (window && !c.prefix && c.sinks < FKV_PAGE_MAX_LEN && seen < span)
        span = seen;
    const int tiles = static_cast<int>((span + kTile - 1) / kTile);
    double best = 0.0;
    p.splits = 1;
    p.chunk = tiles > 0 ? tiles : 1;
    // blocks, and rows of partial results, are counted in a grid dimension
    const bool fits = blocks <= INT32_MAX;
    const int64_t room = INT32_MAX / (blocks > 0 ? blocks : 1);
    const int most_splits = c.n_tok * c.n_q_heads > INT32_MAX ? 1 : static_cast<int>(room < kMaxSplits ? room : kMaxSplits);
    for (int s = 1; s <= most_splits && s <= tiles; ++s) {
        const int chunk = (tiles + s - 1) / s;
        const int64_t waves = (busy * s + slots - 1) / slots;
        const bool in_cluster = p.nt && s > 1 && s <= kMaxCluster && blocks * s <= slots;
        const double join = s == 1 ? 0.0 : in_cluster ? 100.0 : 512.0 + 8.0 * s;
        const double cost = waves * (chunk * kTile + 384.0) + join;
        if (s == 1 || cost < best) {
            best = cost;
            p.splits = (tiles + chunk - 1) / chunk;
            p.chunk = chunk;
        }
    }
    p.cluster = p.nt && p.splits > 1 && p.splits <= kMaxCluster && blocks * p.splits <= slots;
    // A load takes as many units of 16 positions as lie in a page, up to a warp's group
    // (attend4.cu); of 8-bit pages one.
    p.box = 16;
    if (c.pages->format == FKV_UINT4 && p.nt)
        while (p.box < kStep4Keys && c.pages->block % (2 * p.box) == 0)
            p.box *= 2;
    p.workspace = !fits ? -1 : p.splits == 1 || p.cluster ? 0
                : (static_cast<int64_t>(p.splits) * c.n_tok * c.n_q_heads * (c.pages->dim + 1) * 4 + 255) / 256 * 256;
    return p;
}

cudaError_t launch_page_attend(const fkv_ctx *ctx, const fkv_attend &c, const fkv_attend_plan &p, void *ws, const CUtensorMap &mk,
                               const CUtensorMap &mv, cudaStream_t st)
{
    const fkv_pages *pg = c.pages;
    AttendArgs a;
    a.q = c.q, a.out = c.out, a.lse = c.lse, a.pool_k = pg->k, a.pool_v = pg->v;
    a.sb = pg->stride_block, a.sh = pg->stride_head, a.st = pg->stride_pos;
    a.cu = c.cu, a.kv_len = c.kv_len, a.table = c.table;
    a.ks = pg->k_scale, a.vs = pg->v_scale, a.slopes = c.slopes, a.prefix = c.prefix;
    a.status = ctx->d_status;
    a.q_tok = c.q_stride_tok, a.q_head = c.q_stride_head, a.o_tok = c.out_stride_tok, a.o_head = c.out_stride_head;
    a.table_stride = c.table_stride, a.scb = pg->scale_stride_block, a.sch = pg->scale_stride_head;
    a.n_blocks = pg->n_blocks, a.T = c.n_tok;
    a.n_req = static_cast<int>(c.n_req), a.H = pg->n_heads, a.G = c.n_q_heads / pg->n_heads, a.block = pg->block;
    a.width = static_cast<int>(c.width), a.max_new = static_cast<int>(c.max_new), a.max_len = static_cast<int>(c.max_len);
    a.window = window_of(c);
    a.sinks = a.window ? static_cast<int>(c.sinks < FKV_PAGE_MAX_LEN ? c.sinks : FKV_PAGE_MAX_LEN) : 0;
    a.causal = c.causal;
    a.scale = c.scale, a.softcap = c.softcap;
    // (a cap next to float32's largest has a reciprocal of zero: y is zero, f(s) is s)
    a.cap2 = c.softcap * kLog2e, a.cap_inv = c.softcap > 0.0f ? 1.0f / a.cap2 : 0.0f;
    a.div = FastDiv::make(pg->block), a.gdiv = FastDiv::make(a.G);
    a.box = __builtin_ctz(static_cast<unsigned>(p.box)) - 4;
    a.row_tiles = p.row_tiles, a.splits = p.splits, a.chunk = p.chunk, a.cluster = p.cluster;
    a.ws_o = static_cast<float *>(ws);
    a.ws_lse = a.ws_o ? a.ws_o + static_cast<int64_t>(p.splits) * c.n_tok * c.n_q_heads * pg->dim : nullptr;
    if (pg->format == FKV_UINT4) {
        if (pg->dim == 64)
            return c.dtype == FKV_F16 ? step4_as<64, __half>(ctx, a, p.nt, mk, mv, st) : step4_as<64, __nv_bfloat16>(ctx, a, p.nt, mk, mv, st);
        return c.dtype == FKV_F16 ? step4_as<128, __half>(ctx, a, p.nt, mk, mv, st) : step4_as<128, __nv_bfloat16>(ctx, a, p.nt, mk, mv, st);
    }
    const bool i8 = pg->format == FKV_INT8;
    if (pg->dim == 64)
        return i8 ? step_dt<64, FKV_INT8>(ctx, a, c.dtype, p.nt, mk, mv, st) : step_dt<64, FKV_E4M3>(ctx, a, c.dtype, p.nt, mk, mv, st);
    return i8 ? step_dt<128, FKV_INT8>(ctx, a, c.dtype, p.nt, mk, mv, st) : step_dt<128, FKV_E4M3>(ctx, a, c.dtype, p.nt, mk, mv, st);
}
