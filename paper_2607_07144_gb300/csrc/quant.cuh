// Elements to codes of the paged cache and back: what the kernels that write and
// read pages share (paged.cu, append.cu).
#pragma once

#include <type_traits>

#include "paged.cuh"

#ifdef __CUDACC__
namespace fkvd {

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

// The two numbers of a 4-bit row: step in the low half, middle in the high.
__device__ __forceinline__ float step_of(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float middle_of(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// 16 values of a 4-bit row: middle + (code - 7.5) step, whose product is exact in float32.
__device__ __forceinline__ void values16_4bit(const uint2 &v, uint32_t numbers, float *x)
{
    const float step = step_of(numbers), mid = middle_of(numbers);
    const uint32_t w[2] = {v.x, v.y};
#pragma unroll
    for (int i = 0; i < 16; ++i)
        x[i] = fmaf(static_cast<float>(w[i >> 3] >> (4 * (i & 7)) & 15u) - 7.5f, step, mid);
}

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

}  // namespace fkvd
#endif
