// Dropout on its own (qbp_dropout in include/qbp.h).  The mask is made where it is used, forward and backward alike.
#include "qbp_dropout.cuh"

#include <algorithm>

namespace qbp {

constexpr int kDropThreads = 256;

// A thread takes the eight elements of a Philox block, `U` blocks that a thread block's width lies between: their loads are all on their
// way before the first block's generator runs, which needs none of them.  Memory is the bound (4 bytes an element of the halves, and about
// 11 instructions), so what counts is how much of it is asked for at a time: 128 M bf16 elements with one block a thread 115 us.
template <typename T, int U>
__global__ void __launch_bounds__(kDropThreads) dropout_kernel(const T *x, T *y, int64_t n, int vec, const DropoutParams d, const __grid_constant__ PhiloxKeys keys)
{
    const int64_t first = (int64_t)blockIdx.x * kDropThreads * U + threadIdx.x;
    const bool none = d.threshold == 65536u;
    const uint32_t t = none ? 0xFFFFFFFFu : d.threshold << 16;
    pdl_wait();
    Raw8<T> raw[U];
    if (vec && ((int64_t)blockIdx.x + 1) * kDropThreads * U * 8 <= n) {
        const uint4 *src = reinterpret_cast<const uint4 *>(x) + first * (sizeof(T) / 2);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int k = 0; k < (int)(sizeof(T) / 2); ++k) {
                const uint4 *p = src + (int64_t)u * kDropThreads * (sizeof(T) / 2) + k;
                if (sizeof(T) == 4 && vec == 2) { if (k == 0) get32(p, raw[u].w[0], raw[u].w[sizeof(T) / 2 - 1]); }
                else raw[u].w[k] = *p;
            }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t b = first + (int64_t)u * kDropThreads;
            const uint4 w = dropout_block(d, keys, (uint64_t)b);
            float v[8];
            unpack8(raw[u], v);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const uint32_t word = k < 2 ? w.x : k < 4 ? w.y : k < 6 ? w.z : w.w;
                v[k] = ((k & 1) ? word : word << 16) >= t && !none ? __fmul_rn(v[k], d.factor) : 0.0f;
            }
            const Raw8<T> r = pack8<T>(v);
            if (sizeof(T) == 4 && vec == 2) put32(y + b * 8, r.w[0], r.w[sizeof(T) / 2 - 1]);
            else store8(y + b * 8, r, 8, true);
        }
    } else {
        for (int u = 0; u < U; ++u) {
            const int64_t b = first + (int64_t)u * kDropThreads;
            if (b * 8 >= n) break;
            const int here = (int)min((int64_t)8, n - b * 8);
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = k < here ? real_of(x[b * 8 + k]) : 0.0f;
            const uint4 w = dropout_block(d, keys, (uint64_t)b);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = draw_of(w, k) >= d.threshold ? __fmul_rn(v[k], d.factor) : 0.0f;
            store8(y + b * 8, pack8<T>(v), here, false);
        }
    }
}

template <typename T, int U> static void launch_dropout(const void *x, void *y, int64_t n, int vec, const DropoutParams &d, const PhiloxKeys &keys, cudaStream_t st)
{
    const int64_t per_block = (int64_t)kDropThreads * U * 8;
    launch(dropout_kernel<T, U>, (unsigned)((n + per_block - 1) / per_block), kDropThreads, 0, st, (const T *)x, (T *)y, n, vec, d, keys);
}
// Blocks of eight a thread takes: four of the halves and two of fp32 (64 bytes) where that still fills the SMs twice.
template <typename T> static void launch_dropout(const void *x, void *y, int64_t n, int vec, const DropoutParams &d, const PhiloxKeys &keys, cudaStream_t st)
{
    constexpr int many = sizeof(T) == 2 ? 4 : 2;
    if (n >= (int64_t)2 * 8 * kDropThreads * 8 * many * sm_count()) launch_dropout<T, many>(x, y, n, vec, d, keys, st);
    else launch_dropout<T, 1>(x, y, n, vec, d, keys, st);
}

extern "C" __attribute__((visibility("default"))) int qbp_dropout(const void *x, int dtype, int64_t n, float p, uint64_t seed, uint32_t tensor_id,
                                                                  uint64_t index_base, void *y, void *stream)
{
    cudaStream_t st = (cudaStream_t)stream;
    if (!dtype_ok(dtype)) return fail(QBP_ERR_INVALID_ARG, "dropout: dtype %d", dtype);
    if (n < 0) return fail(QBP_ERR_INVALID_ARG, "dropout: %lld elements", (long long)n);
    if (!(p >= 0.0f && p <= 1.0f)) return fail(QBP_ERR_INVALID_ARG, "dropout: p = %g is not in [0, 1]", (double)p);
    if (index_base % 8) return fail(QBP_ERR_INVALID_ARG, "dropout: index_base %llu is not a multiple of 8", (unsigned long long)index_base);
    if (n == 0) return QBP_OK;
    if (!x || !y || !aligned_to(x, dtype_size(dtype)) || !aligned_to(y, dtype_size(dtype))) return fail(QBP_ERR_INVALID_ARG, "dropout: x or y is NULL or misaligned");
    const DropoutParams d = dropout_params(p, tensor_id, index_base);
    const PhiloxKeys keys = philox_keys_host(seed);
    const int vec = aligned_to(x, 32) && aligned_to(y, 32) ? 2 : aligned16(x) && aligned16(y) ? 1 : 0;
    if (n > ((int64_t)1 << 41)) return fail(QBP_ERR_UNSUPPORTED_SHAPE, "dropout: %lld elements", (long long)n);
    QBP_TRACE_BEGIN(st);
    QBP_FOR_DTYPE(dtype, T, launch_dropout<T>(x, y, n, vec, d, keys, st));
    QBP_LAUNCH_OK("dropout_kernel");
    return QBP_OK;
}

}  // namespace qbp
