// Device helpers shared by the kernels of the paged 8-bit K/V cache.
#pragma once

#include "fkv_internal.h"

// Smallest scale of a page (2^-100): attention works with a value scale's
// logarithm and reciprocal, and a page of zeros has to have both.
#define FKV_PAGE_MIN_SCALE 7.888609052210118e-31f
// And the largest, 2^100: its share of a sum of weights (attend.cuh) is one that
// float32 holds.
#define FKV_PAGE_MAX_SCALE 1.2676506002282294e30f

#ifdef __CUDACC__
// Launch `kernel` so that its blocks may be scheduled while the stream's
// previous kernel ends; it waits (griddepcontrol.wait) before it reads what that
// one wrote.
template <typename... Args, typename... Given>
cudaError_t launch_after(void (*kernel)(Args...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, const Given &...args)
{
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid, cfg.blockDim = block, cfg.dynamicSmemBytes = smem, cfg.stream = st;
    cfg.attrs = &at, cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

namespace fkvd {

// Two e4m3 codes (the lower byte first) as two fp16, exactly.
__device__ __forceinline__ __half2 e4m3x2_half2(uint16_t w)
{
    uint32_t d;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(d) : "h"(w));
    return *reinterpret_cast<__half2 *>(&d);
}

// Four 8-bit codes as fp16, exactly: (w0, w1) and (w2, w3).  An int8 code b is
// the fp16 number 1024 + (b + 128) by its bits, less 1152.
template <int FMT> __device__ __forceinline__ void codes4_half(uint32_t w, uint32_t &lo, uint32_t &hi)
{
    if (FMT == FKV_INT8) {
        const uint32_t x = w ^ 0x80808080u;
        const __half2 bias = __half2half2(__ushort_as_half(0x6480));
        uint32_t a = __byte_perm(x, 0x64646464u, 0x4140), b = __byte_perm(x, 0x64646464u, 0x4342);
        __half2 ha = __hsub2(*reinterpret_cast<__half2 *>(&a), bias), hb = __hsub2(*reinterpret_cast<__half2 *>(&b), bias);
        lo = *reinterpret_cast<uint32_t *>(&ha);
        hi = *reinterpret_cast<uint32_t *>(&hb);
    } else {
        asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\t"
            "cvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
            : "=r"(lo), "=r"(hi)
            : "r"(w));
    }
}

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ float lg2(float x)
{
    float y;
    asm("lg2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

}  // namespace fkvd
#endif
