// pf_ops.cuh -- device helpers shared by the decode-layer operators (planfront_ops.h): number formats, asynchronous
// copies, the 16-bit matrix instruction.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "pf_internal.cuh"
#include "planfront_ops.h"

namespace pf {

constexpr float kE4m3Max = 448.f;
constexpr float kMinScale = 7.888609052210118e-31f;   // 2^-100

// ------------------------------------------------------------------ number formats
// two fp32 -> two e4m3 bytes (nearest even, saturated; NaN stays NaN), `lo` in the lower byte
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi)
{
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d)
{
    return e4m3x2(a, b) | (e4m3x2(c, d) << 16);
}
// two e4m3 bytes -> two fp16 (exact)
__device__ __forceinline__ uint32_t f16x2_of_e4m3x2(uint32_t v)
{
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)v));
    return r;
}
__device__ __forceinline__ uint32_t f16x2_of(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t bf16x2_of(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float2 f32x2_of_bf16x2(uint32_t v)
{
    return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xFFFF0000u));
}
__device__ __forceinline__ float2 f32x2_of_f16x2(uint32_t v)
{
    return __half22float2(*reinterpret_cast<__half2 *>(&v));
}

// 8 elements of type T <-> fp32
struct Bf16 { uint16_t bits; };
struct F16 { uint16_t bits; };
template <typename T> __device__ __forceinline__ float2 pair_to_f32(uint32_t v);
template <> __device__ __forceinline__ float2 pair_to_f32<Bf16>(uint32_t v) { return f32x2_of_bf16x2(v); }
template <> __device__ __forceinline__ float2 pair_to_f32<F16>(uint32_t v) { return f32x2_of_f16x2(v); }
template <typename T> __device__ __forceinline__ uint32_t pair_of_f32(float a, float b);
template <> __device__ __forceinline__ uint32_t pair_of_f32<Bf16>(float a, float b) { return bf16x2_of(a, b); }
template <> __device__ __forceinline__ uint32_t pair_of_f32<F16>(float a, float b) { return f16x2_of(a, b); }

// ------------------------------------------------------------------ the cache's scales
// the exponent of the least power of two >= amax / 448, in [-100, 118]; amax >= 0, infinity included
__device__ __forceinline__ int scale_exponent(float amax)
{
    if (!(amax > 0.f)) return -100;
    const uint32_t b = __float_as_uint(amax);
    // amax = 1.m * 2^(E - 127), 448 = 1.75 * 2^8; a subnormal amax reads E = 0 and lands below the floor either way
    const int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return max(-100, min(118, e));
}
__device__ __forceinline__ float pow2f(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // -126 <= e <= 127

// ------------------------------------------------------------------ asynchronous copies, global -> shared
__device__ __forceinline__ uint32_t smem_addr(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
// 16 bytes, of which the first `bytes` (0 or 16) are read and the rest are zero; past L1
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, uint32_t bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t dst, const void *src)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ uint4 lds128(uint32_t a)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t a)
{
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
    return v;
}

// ------------------------------------------------------------------ matrix instruction
// D[16 x 8] += A[16 x 16] B[16 x 8], fp32 sums.  Lane 4 g + q holds A rows g and g + 8, columns 2q, 2q + 1 (a0, a1) and 2q + 8,
// 2q + 9 (a2, a3); B rows 2q, 2q + 1 (b0) and 2q + 8, 2q + 9 (b1) of column g; D rows g (c0, c1) and g + 8 (c2, c3), columns
// 2q, 2q + 1.  The order of the 16 summed indices is free as long as A and B agree, which the layouts here use: a lane's
// four A columns of a step stand for four neighbouring elements of a row.
template <typename T>
__device__ __forceinline__ void mma16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma16<F16>(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma16<Bf16>(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// ------------------------------------------------------------------ host
inline bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }
// number of SMs of the current device; PF_ECUDA if it cannot be read
inline int current_sm_count(int *device, int *sm_count)
{
    PF_CUDA_TRY(cudaGetDevice(device), "cudaGetDevice");
    PF_CUDA_TRY(cudaDeviceGetAttribute(sm_count, cudaDevAttrMultiProcessorCount, *device), "cudaDeviceGetAttribute");
    return PF_OK;
}

inline bool kv_cache_ok(const pf_kv_cache_t *c)
{
    return c && c->n_pages > 0 && c->n_kv > 0 && (c->page == 16 || c->page == 32 || c->page == 64 || c->page == 128) &&
           (c->hd == 64 || c->hd == 128) && c->d_k && c->d_v && c->d_k_scale && c->d_v_scale && aligned16(c->d_k) &&
           aligned16(c->d_v) && (uintptr_t)c->d_k_scale % 4 == 0 && (uintptr_t)c->d_v_scale % 4 == 0;
}

}  // namespace pf
