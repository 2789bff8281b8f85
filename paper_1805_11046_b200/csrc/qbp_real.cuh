// Real-valued tensors in fp32, bf16 or fp16 (qbp_dtype): what the 8-bit floating-point quantiser, the joins and the
// dropout read and write.  Arithmetic is fp32 whatever the type; a result is rounded once, as it is stored.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "qbp_common.cuh"

namespace qbp {

inline size_t dtype_size(int dtype) { return dtype == QBP_F32 ? 4 : 2; }
inline bool dtype_ok(int dtype) { return dtype == QBP_F32 || dtype == QBP_BF16 || dtype == QBP_F16; }
inline bool aligned_to(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// Runs `call` with T the element type of `dtype` (checked by the caller).
#define QBP_FOR_DTYPE(dtype, T, call)                                  \
    do {                                                               \
        if ((dtype) == QBP_F32) { using T = float; call; }             \
        else if ((dtype) == QBP_BF16) { using T = __nv_bfloat16; call; } \
        else { using T = __half; call; }                               \
    } while (0)

#ifdef __CUDACC__

__device__ __forceinline__ float real_of(float v) { return v; }
__device__ __forceinline__ float real_of(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float real_of(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T real_to(float v);
template <> __device__ __forceinline__ float real_to<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 real_to<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half real_to<__half>(float v) { return __float2half_rn(v); }

// Eight consecutive elements as they lie in memory: 32 bytes of fp32 or 16 of the halves.
template <typename T> struct Raw8 { uint4 w[sizeof(T) / 2]; };
template <typename T> __device__ __forceinline__ void unpack8(const Raw8<T> &r, float (&v)[8])
{
    const T *e = reinterpret_cast<const T *>(r.w);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = real_of(e[i]);
}
// Two values to two halves in one conversion, or as they are.
__device__ __forceinline__ void put_two(float *e, float a, float b) { e[0] = a; e[1] = b; }
__device__ __forceinline__ void put_two(__nv_bfloat16 *e, float a, float b) { *reinterpret_cast<__nv_bfloat162 *>(e) = __floats2bfloat162_rn(a, b); }
__device__ __forceinline__ void put_two(__half *e, float a, float b) { *reinterpret_cast<__half2 *>(e) = __floats2half2_rn(a, b); }
template <typename T> __device__ __forceinline__ Raw8<T> pack8(const float (&v)[8])
{
    Raw8<T> r;
    T *e = reinterpret_cast<T *>(r.w);
#pragma unroll
    for (int i = 0; i < 8; i += 2) put_two(e + i, v[i], v[i + 1]);
    return r;
}

// The first `n` (at most 8) of eight elements at p, zeros behind them; vec: p is on a 16-byte boundary.
template <typename T> __device__ __forceinline__ Raw8<T> load8(const T *p, int n, bool vec)
{
    Raw8<T> r;
    if (vec && n >= 8) {
#pragma unroll
        for (int i = 0; i < (int)(sizeof(T) / 2); ++i) r.w[i] = __ldg(reinterpret_cast<const uint4 *>(p) + i);
    } else {
        T *e = reinterpret_cast<T *>(r.w);
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = i < n ? __ldg(p + i) : real_to<T>(0.0f);
    }
    return r;
}
template <typename T> __device__ __forceinline__ void store8(T *p, const Raw8<T> &r, int n, bool vec)
{
    if (vec && n >= 8) {
#pragma unroll
        for (int i = 0; i < (int)(sizeof(T) / 2); ++i) reinterpret_cast<uint4 *>(p)[i] = r.w[i];
    } else {
        const T *e = reinterpret_cast<const T *>(r.w);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = e[i];
    }
}

// 32 bytes at a time, on a 32-byte boundary: eight fp32 of a lane in one access.  (As two of 16 bytes each access asks for half of 32
// sectors.)
__device__ __forceinline__ void put32(void *p, const uint4 &a, const uint4 &b)
{
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b.x), "r"(b.y), "r"(b.z), "r"(b.w)
                 : "memory");
}
__device__ __forceinline__ void get32(const void *p, uint4 &a, uint4 &b)
{
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(a.x), "=r"(a.y), "=r"(a.z), "=r"(a.w), "=r"(b.x), "=r"(b.y), "=r"(b.z), "=r"(b.w) : "l"(p) : "memory");
}

#endif  // __CUDACC__
}  // namespace qbp
