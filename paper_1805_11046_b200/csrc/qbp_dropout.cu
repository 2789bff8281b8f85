// Dropout on its own (qbp_dropout in include/qbp.h).  The mask is made where it is used, forward and backward alike.
#include "qbp_dropout.cuh"

#include <algorithm>

namespace qbp {

constexpr int kDropThreads = 256;

// A thread takes the eight elements of one Philox block.
template <typename T>
__global__ void __launch_bounds__(kDropThreads) dropout_kernel(const T *x, T *y, int64_t n, int vec, const DropoutParams d, const __grid_constant__ PhiloxKeys keys)
{
    pdl_wait();
    for (int64_t b = (int64_t)blockIdx.x * kDropThreads + threadIdx.x; b * 8 < n; b += (int64_t)gridDim.x * kDropThreads) {
        const int here = (int)min((int64_t)8, n - b * 8);
        const Raw8<T> raw = load8(x + b * 8, here, vec != 0);
        const uint4 w = dropout_block(d, keys, (uint64_t)b);
        float v[8];
        unpack8(raw, v);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = draw_of(w, k) >= d.threshold ? __fmul_rn(v[k], d.factor) : 0.0f;
        store8(y + b * 8, pack8<T>(v), here, vec != 0);
    }
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
    const int vec = aligned16(x) && aligned16(y) ? 1 : 0;
    const int64_t blocks = ((n + 7) / 8 + kDropThreads - 1) / kDropThreads;
    const unsigned grid = (unsigned)std::min<int64_t>(blocks, 0x7FFFFFFF);
    QBP_TRACE_BEGIN(st);
    QBP_FOR_DTYPE(dtype, T, launch(dropout_kernel<T>, grid, kDropThreads, 0, st, (const T *)x, (T *)y, n, vec, d, keys));
    QBP_LAUNCH_OK("dropout_kernel");
    return QBP_OK;
}

}  // namespace qbp
