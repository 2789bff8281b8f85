// The join between two blocks of a residual network and its gradients (qbp_resnorm_fwd / _bwd in include/qbp.h): norm after a
// block, gate, dropout, residual stream and the norm before the next block, in one pass over the rows.
//
// A row is held in registers by the threads of one group: a warp of a block's eight for rows of up to 1024 columns, the whole
// block beyond; a thread has CH chunks of eight neighbouring columns.  The two sums over a row (of b^2 and of r^2; backwards of the
// gradients' projections on r and b) each cost one exchange between the group's threads, and nothing is read twice.
// Backwards a thread keeps the sums over its rows for its columns (dw_post, dgate, dw_pre) in registers, a block leaves one
// partial row of each, and a second kernel adds these up in a fixed order.
#include "qbp_dropout.cuh"

#include <algorithm>

namespace qbp {

constexpr int kJoinWarpRows = 8;                    // rows of a block whose groups are warps
constexpr int64_t kJoinMaxCols = QBP_RESNORM_MAX_COLS;

struct JoinParams {
    int64_t rows, cols, gate_rows;
    const void *x, *b; const float *w_post, *gate, *w_pre;
    void *r, *h; float *rstd_post, *rstd_pre;
    float eps, alpha, inv_cols;
    int post, pre, drop, vec_x, vec_b, vec_w;
    DropoutParams d;
};

struct JoinBwdParams {
    int64_t rows, cols, gate_rows, gates, splits, split_rows;    // an item: `split_rows` rows of a gate (the last one fewer)
    const void *dr, *dh, *b, *r; const float *rstd_post, *rstd_pre, *w_post, *gate, *w_pre;
    void *dx, *db; float *part_post, *part_gate, *part_pre;
    float alpha, inv_cols;
    int post, pre, drop, vec_x, vec_b, vec_w, sum_post, sum_gate, sum_pre;
    DropoutParams d;
};

// Sum over the threads of a row's group; every thread gets it.  WARP: the group is a warp.  `turn` alternates between the two
// halves of the scratch, so that one barrier per sum is enough.
template <bool WARP> __device__ __forceinline__ float group_sum(float v, float (&scratch)[2][32], int turn)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    if (WARP) return v;
    if ((threadIdx.x & 31) == 0) scratch[turn][threadIdx.x >> 5] = v;
    __syncthreads();
    float s = 0.0f;
    for (unsigned w = 0; w < blockDim.x / 32; ++w) s += scratch[turn][w];
    return s;
}

// Eight fp32 parameters of neighbouring columns (absent: ones).
__device__ __forceinline__ void load_params(const float *p, int64_t at, int n, int vec, float (&v)[8])
{
    if (!p) {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = 1.0f;
    } else {
        unpack8(load8(p + at, n, vec != 0), v);
    }
}
__device__ __forceinline__ void keep_factors(const DropoutParams &d, const PhiloxKeys &keys, int64_t element, float (&k8)[8])
{
    const uint4 w = dropout_draws8(d, keys, (uint64_t)element);
#pragma unroll
    for (int k = 0; k < 8; ++k) k8[k] = draw_of(w, k) >= d.threshold ? d.factor : 0.0f;
}

template <typename TX, typename TB, int CH, bool WARP>
__global__ void __launch_bounds__(WARP ? 32 * kJoinWarpRows : 512) join_fwd_kernel(const __grid_constant__ JoinParams P, const __grid_constant__ PhiloxKeys keys)
{
    __shared__ float scratch[2][32];
    const int group = WARP ? 32 : blockDim.x, t = WARP ? (threadIdx.x & 31) : threadIdx.x;
    const int64_t step = WARP ? (int64_t)gridDim.x * kJoinWarpRows : gridDim.x;
    pdl_wait();
    for (int64_t row = WARP ? (int64_t)blockIdx.x * kJoinWarpRows + (threadIdx.x >> 5) : blockIdx.x; row < P.rows; row += step) {
        const int64_t base = row * P.cols, grow = P.gate_rows ? row / P.gate_rows : 0;
        Raw8<TX> xr[CH]; Raw8<TB> br[CH];
        int n[CH];
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int64_t c = 8ll * (t + k * group);
            n[k] = (int)max((int64_t)0, min((int64_t)8, P.cols - c));
            xr[k] = load8(static_cast<const TX *>(P.x) + (n[k] ? base + c : 0), n[k], P.vec_x != 0);
            if (P.b) br[k] = load8(static_cast<const TB *>(P.b) + (n[k] ? base + c : 0), n[k], P.vec_b != 0);
        }
        float rstd = 1.0f;
        if (P.post) {
            float s = 0.0f;
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                float v[8];
                unpack8(br[k], v);
#pragma unroll
                for (int e = 0; e < 8; ++e) s = fmaf(v[e], v[e], s);
            }
            rstd = 1.0f / sqrtf(group_sum<WARP>(s, scratch, 0) * P.inv_cols + P.eps);
            if (P.rstd_post && t == 0) P.rstd_post[row] = rstd;
        }
        float s2 = 0.0f;
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int64_t c = 8ll * (t + k * group);
            float x[8];
            unpack8(xr[k], x);
            if (P.b) {
                float b[8], w[8], g[8], m[8];
                unpack8(br[k], b);
                load_params(P.post ? P.w_post : nullptr, c, n[k], P.vec_w, w);
                load_params(P.gate, grow * P.cols + c, n[k], P.vec_w, g);
                if (P.drop) keep_factors(P.d, keys, base + c, m);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float v = P.post ? b[e] * rstd * w[e] : b[e];
                    if (P.drop) v = m[e] != 0.0f ? v * m[e] : 0.0f;
                    x[e] = P.alpha * x[e] + g[e] * v;
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = P.alpha * x[e];
            }
            xr[k] = pack8<TX>(x);
            if (P.r && n[k]) store8(static_cast<TX *>(P.r) + base + c, xr[k], n[k], P.vec_x != 0);
            unpack8(xr[k], x);
#pragma unroll
            for (int e = 0; e < 8; ++e) s2 = e < n[k] ? fmaf(x[e], x[e], s2) : s2;
        }
        if (P.pre) {
            const float rstd2 = 1.0f / sqrtf(group_sum<WARP>(s2, scratch, 1) * P.inv_cols + P.eps);
            if (P.rstd_pre && t == 0) P.rstd_pre[row] = rstd2;
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                const int64_t c = 8ll * (t + k * group);
                float x[8], w[8];
                unpack8(xr[k], x);
                load_params(P.w_pre, c, n[k], P.vec_w, w);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = x[e] * rstd2 * w[e];
                if (n[k]) store8(static_cast<TB *>(P.h) + base + c, pack8<TB>(x), n[k], P.vec_b != 0);
            }
        }
        if (!WARP && P.pre != P.post) __syncthreads();   // one sum a row: the next row's writes the half that this one's may still be read from
    }
}

template <typename TX, typename TB, int CH, bool WARP>
__global__ void __launch_bounds__(WARP ? 32 * kJoinWarpRows : 512) join_bwd_kernel(const __grid_constant__ JoinBwdParams P, const __grid_constant__ PhiloxKeys keys)
{
    extern __shared__ float fold[];                  // WARP: [kJoinWarpRows][cols rounded up to 8], the warps' sums
    __shared__ float scratch[2][32];
    const int group = WARP ? 32 : blockDim.x, t = WARP ? (threadIdx.x & 31) : threadIdx.x, sub = WARP ? threadIdx.x >> 5 : 0;
    const int subs = WARP ? kJoinWarpRows : 1;
    const int64_t pitch = (P.cols + 7) / 8 * 8;
    float a_post[CH][8] = {}, a_gate[CH][8] = {}, a_pre[CH][8] = {};
    // A thread's sums of one kind to the block's partial row (and back to zero).
    const auto leave = [&](float (&a)[CH][8], float *out) {
        if (WARP) {
            __syncthreads();
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                const int64_t c = 8ll * (t + k * group);
                if (c < P.cols) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) fold[sub * pitch + c + e] = a[k][e];
                }
            }
            __syncthreads();
            for (int64_t c = threadIdx.x; c < P.cols; c += blockDim.x) {
                float s = 0.0f;
#pragma unroll
                for (int q = 0; q < kJoinWarpRows; ++q) s += fold[q * pitch + c];
                out[c] = s;
            }
        } else {
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                const int64_t c = 8ll * (t + k * group);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (c + e < P.cols) out[c + e] = a[k][e];
            }
        }
#pragma unroll
        for (int k = 0; k < CH; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) a[k][e] = 0.0f;
    };
    pdl_wait();
    for (int64_t item = blockIdx.x; item < P.gates * P.splits; item += gridDim.x) {
        const int64_t g = item / P.splits, first = g * P.gate_rows + item % P.splits * P.split_rows;
        const int64_t end = min(min(first + P.split_rows, (g + 1) * P.gate_rows), P.rows);
        for (int64_t row = first + sub; row < end; row += subs) {
            const int64_t base = row * P.cols;
            Raw8<TX> gr[CH], rr[CH]; Raw8<TB> hr[CH], br[CH];
            int n[CH];
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                const int64_t c = 8ll * (t + k * group);
                n[k] = (int)max((int64_t)0, min((int64_t)8, P.cols - c));
                const int64_t at = n[k] ? base + c : 0;
                gr[k] = load8(static_cast<const TX *>(P.dr) + (P.dr ? at : 0), P.dr ? n[k] : 0, P.vec_x != 0);
                if (P.pre) { rr[k] = load8(static_cast<const TX *>(P.r) + at, n[k], P.vec_x != 0); hr[k] = load8(static_cast<const TB *>(P.dh) + at, n[k], P.vec_b != 0); }
                if (P.b) br[k] = load8(static_cast<const TB *>(P.b) + at, n[k], P.vec_b != 0);
            }
            float rstd2 = 0.0f, mean2 = 0.0f;
            if (P.pre) {
                rstd2 = P.rstd_pre[row];
                float s = 0.0f;
#pragma unroll
                for (int k = 0; k < CH; ++k) {
                    float h[8], r[8], w[8];
                    unpack8(hr[k], h); unpack8(rr[k], r);
                    load_params(P.w_pre, 8ll * (t + k * group), n[k], P.vec_w, w);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float rh = r[e] * rstd2;
                        a_pre[k][e] = fmaf(h[e], rh, a_pre[k][e]);
                        s = fmaf(h[e] * w[e], rh, s);
                    }
                }
                mean2 = group_sum<WARP>(s, scratch, 0) * P.inv_cols;
            }
            const float rstd1 = P.post ? P.rstd_post[row] : 1.0f;
            float s1 = 0.0f;
            float v8[CH][8];                             // v w_post of the row (without a post norm: v)
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                const int64_t c = 8ll * (t + k * group);
                float R[8];
                unpack8(gr[k], R);
                if (P.pre) {
                    float h[8], r[8], w[8];
                    unpack8(hr[k], h); unpack8(rr[k], r);
                    load_params(P.w_pre, c, n[k], P.vec_w, w);
#pragma unroll
                    for (int e = 0; e < 8; ++e) R[e] += rstd2 * (h[e] * w[e] - r[e] * rstd2 * mean2);
                }
                if (P.b) {
                    float b[8], w[8], gt[8], m[8];
                    unpack8(br[k], b);
                    load_params(P.post ? P.w_post : nullptr, c, n[k], P.vec_w, w);
                    load_params(P.gate, g * P.cols + c, n[k], P.vec_w, gt);
                    if (P.drop) keep_factors(P.d, keys, base + c, m);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float bh = b[e] * rstd1, q = P.drop ? m[e] : 1.0f;
                        const float v = q != 0.0f ? R[e] * gt[e] * q : 0.0f;
                        a_gate[k][e] += q != 0.0f ? R[e] * (bh * w[e] * q) : 0.0f;
                        a_post[k][e] = fmaf(v, bh, a_post[k][e]);
                        v8[k][e] = v * w[e];
                        s1 = fmaf(v8[k][e], bh, s1);
                    }
                }
                if (P.dx && n[k]) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) R[e] *= P.alpha;
                    store8(static_cast<TX *>(P.dx) + base + c, pack8<TX>(R), n[k], P.vec_x != 0);
                }
            }
            if (P.b) {
                const float mean1 = P.post ? group_sum<WARP>(s1, scratch, 1) * P.inv_cols : 0.0f;
                if (P.db) {
#pragma unroll
                    for (int k = 0; k < CH; ++k) {
                        if (P.post) {
                            float b[8];
                            unpack8(br[k], b);
#pragma unroll
                            for (int e = 0; e < 8; ++e) v8[k][e] = rstd1 * (v8[k][e] - b[e] * rstd1 * mean1);
                        }
                        if (n[k]) store8(static_cast<TB *>(P.db) + base + 8ll * (t + k * group), pack8<TB>(v8[k]), n[k], P.vec_b != 0);
                    }
                }
            }
            if (!WARP && P.pre != P.post) __syncthreads();   // one sum a row: the next row's writes the half that this one's may still be read from
        }
        if (P.sum_gate) leave(a_gate, P.part_gate + item * P.cols);
    }
    if (P.sum_post) leave(a_post, P.part_post + (int64_t)blockIdx.x * P.cols);
    if (P.sum_pre) leave(a_pre, P.part_pre + (int64_t)blockIdx.x * P.cols);
}

// out[o][c] = sum over `count` partial rows in [outs][count][cols], in a fixed order: sixteen threads of a column take every sixteenth, then
// the sixteen are added up.
struct JoinSum { const float *part; float *out; int64_t outs, count; };
struct JoinSums { JoinSum j[3]; int64_t cols; };
constexpr int kSumHigh = 16;
__global__ void __launch_bounds__(32 * kSumHigh) join_sum_kernel(const __grid_constant__ JoinSums S)
{
    __shared__ float s_part[kSumHigh][33];
    const JoinSum &j = S.j[blockIdx.z];
    const int lane = threadIdx.x & 31, high = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;
    pdl_wait();
    for (int64_t o = blockIdx.y; o < j.outs; o += gridDim.y) {
        float s = 0.0f;
        if (c < S.cols) {
            const float *p = j.part + o * j.count * S.cols + c;
#pragma unroll 4
            for (int64_t k = high; k < j.count; k += kSumHigh) s += p[k * S.cols];
        }
        s_part[high][lane] = s;
        __syncthreads();
        if (high == 0 && c < S.cols) {
            float v = 0.0f;
#pragma unroll
            for (int k = 0; k < kSumHigh; ++k) v += s_part[k][lane];
            j.out[o * S.cols + c] = v;
        }
        __syncthreads();
    }
}

// ================================================================= host side
struct JoinShape { int ch, threads; bool warp; };
static JoinShape join_shape(int64_t cols)
{
    const int64_t chunks = (cols + 7) / 8;
    if (chunks <= 32) return {1, 32 * kJoinWarpRows, true};
    if (chunks <= 64) return {2, 32 * kJoinWarpRows, true};
    if (chunks <= 128) return {4, 32 * kJoinWarpRows, true};
    if (chunks <= 256) return {2, 128, false};
    if (chunks <= 512) return {2, 256, false};
    if (chunks <= 1024) return {2, 512, false};
    return {4, 512, false};
}

#define QBP_FOR_JOIN(shape, CH, WARP, call)                                                          \
    do {                                                                                             \
        if ((shape).warp) {                                                                          \
            constexpr bool WARP = true;                                                              \
            if ((shape).ch == 1) { constexpr int CH = 1; call; }                                     \
            else if ((shape).ch == 2) { constexpr int CH = 2; call; }                                \
            else { constexpr int CH = 4; call; }                                                     \
        } else {                                                                                     \
            constexpr bool WARP = false;                                                             \
            if ((shape).ch == 2) { constexpr int CH = 2; call; }                                     \
            else { constexpr int CH = 4; call; }                                                     \
        }                                                                                            \
    } while (0)

static int check_join(const qbp_resnorm_desc *d, const char *name, const void *b, const float *gate, const float *w_post, const float *w_pre)
{
    if (!d) return fail(QBP_ERR_INVALID_ARG, "%s: NULL descriptor", name);
    if (!dtype_ok(d->x_dtype) || !dtype_ok(d->b_dtype)) return fail(QBP_ERR_INVALID_ARG, "%s: dtypes %d and %d", name, d->x_dtype, d->b_dtype);
    if (d->rows < 0 || d->cols < 0 || d->gate_rows < 0) return fail(QBP_ERR_INVALID_ARG, "%s: rows %lld, cols %lld, gate_rows %lld", name, (long long)d->rows, (long long)d->cols, (long long)d->gate_rows);
    if (d->cols > kJoinMaxCols) return fail(QBP_ERR_UNSUPPORTED_SHAPE, "%s: %lld columns, at most %lld", name, (long long)d->cols, (long long)kJoinMaxCols);
    if (!(d->eps >= 0.0f) || !(d->p >= 0.0f && d->p <= 1.0f) || std::isinf(d->eps)) return fail(QBP_ERR_INVALID_ARG, "%s: eps %g, p %g", name, (double)d->eps, (double)d->p);
    if (d->index_base % 8) return fail(QBP_ERR_INVALID_ARG, "%s: index_base %llu is not a multiple of 8", name, (unsigned long long)d->index_base);
    if (!b && (d->post || gate || d->p > 0.0f)) return fail(QBP_ERR_INVALID_ARG, "%s: a norm after, a gate or dropout without a block output", name);
    for (const float *w : {gate, w_post, w_pre})
        if (!aligned_to(w, 4)) return fail(QBP_ERR_INVALID_ARG, "%s: misaligned parameters", name);
    return QBP_OK;
}
static bool real_ok(const void *p, int dtype) { return p && aligned_to(p, dtype_size(dtype)); }
static bool rows_vec(const void *p, int dtype, int64_t cols) { return aligned16(p) && cols * (int64_t)dtype_size(dtype) % 16 == 0; }
static int64_t join_gates(const qbp_resnorm_desc *d) { return d->gate_rows ? (d->rows + d->gate_rows - 1) / d->gate_rows : 1; }

extern "C" __attribute__((visibility("default"))) int qbp_resnorm_fwd(const qbp_resnorm_desc *d, const void *x, const void *b, const float *w_post,
                                                                      const float *gate, const float *w_pre, void *r, void *h, float *rstd_post,
                                                                      float *rstd_pre, void *stream)
{
    cudaStream_t st = (cudaStream_t)stream;
    int rc = check_join(d, "resnorm_fwd", b, gate, w_post, w_pre);
    if (rc) return rc;
    if (d->rows == 0 || d->cols == 0) return QBP_OK;
    if (!real_ok(x, d->x_dtype) || (b && !real_ok(b, d->b_dtype)) || (r && !real_ok(r, d->x_dtype)) || (d->pre && !real_ok(h, d->b_dtype)))
        return fail(QBP_ERR_INVALID_ARG, "resnorm_fwd: a tensor is NULL or misaligned");
    if (!r && (b || d->alpha != 1.0f)) return fail(QBP_ERR_INVALID_ARG, "resnorm_fwd: r may be NULL only where it is x");
    if (!r && !d->pre) return fail(QBP_ERR_INVALID_ARG, "resnorm_fwd: no output wanted");
    JoinParams P{};
    P.rows = d->rows; P.cols = d->cols; P.gate_rows = gate ? d->gate_rows : 0;
    P.x = x; P.b = b; P.w_post = w_post; P.gate = gate; P.w_pre = w_pre; P.r = r; P.h = h; P.rstd_post = rstd_post; P.rstd_pre = rstd_pre;
    P.eps = d->eps; P.alpha = d->alpha; P.inv_cols = (float)(1.0 / (double)d->cols);
    P.post = d->post ? 1 : 0; P.pre = d->pre ? 1 : 0;
    P.vec_x = rows_vec(x, d->x_dtype, d->cols) && (!r || aligned16(r)) ? 1 : 0;
    P.vec_b = rows_vec(b, d->b_dtype, d->cols) && (!h || aligned16(h)) ? 1 : 0;
    P.vec_w = aligned16(w_post) && aligned16(gate) && aligned16(w_pre) && d->cols % 4 == 0 ? 1 : 0;
    P.d = dropout_params(d->p, d->tensor_id, d->index_base);
    P.drop = P.d.threshold ? 1 : 0;
    const PhiloxKeys keys = philox_keys_host(d->seed);
    const JoinShape s = join_shape(d->cols);
    const int64_t want = s.warp ? (d->rows + kJoinWarpRows - 1) / kJoinWarpRows : d->rows;
    const unsigned grid = (unsigned)std::min<int64_t>(want, 8ll * sm_count());
    QBP_TRACE_BEGIN(st);
    QBP_FOR_DTYPE(d->x_dtype, TX, QBP_FOR_DTYPE(d->b_dtype, TB, QBP_FOR_JOIN(s, CH, WARP, (launch(join_fwd_kernel<TX, TB, CH, WARP>, grid, s.threads, 0, st, P, keys)))));
    QBP_LAUNCH_OK("join_fwd_kernel");
    return QBP_OK;
}

// How the backward pass cuts the rows: `blocks` blocks, each gate in `splits` items.
struct JoinCut { int64_t blocks, splits, split_rows, gates, gate_rows; };
static JoinCut join_cut(const qbp_resnorm_desc *d, bool per_gate)
{
    JoinCut c;
    const JoinShape s = join_shape(d->cols);
    c.gates = per_gate ? join_gates(d) : 1;
    c.gate_rows = per_gate && d->gate_rows ? d->gate_rows : std::max<int64_t>(d->rows, 1);
    const int64_t most = 2ll * sm_count();
    // a warp's row costs a quarter of a block's, and a block of warps takes eight at a time
    const int64_t few = s.warp ? 2 * kJoinWarpRows : 2;
    c.splits = std::max<int64_t>(1, std::min((most + c.gates - 1) / c.gates, (c.gate_rows + few - 1) / few));
    c.split_rows = (c.gate_rows + c.splits - 1) / c.splits;
    c.splits = (c.gate_rows + c.split_rows - 1) / c.split_rows;
    c.blocks = std::min(most, c.gates * c.splits);
    return c;
}

extern "C" __attribute__((visibility("default"))) size_t qbp_resnorm_bwd_workspace_bytes(const qbp_resnorm_desc *d)
{
    if (!d || d->rows <= 0 || d->cols <= 0) return 256;
    size_t most = 0;
    for (bool per_gate : {false, true}) {
        const JoinCut c = join_cut(d, per_gate);
        most = std::max(most, 2 * align_up((size_t)(c.blocks * d->cols) * 4, 256) + align_up((size_t)(c.gates * c.splits * d->cols) * 4, 256));
    }
    return 256 + most;
}

extern "C" __attribute__((visibility("default"))) int qbp_resnorm_bwd(const qbp_resnorm_desc *d, const void *dr, const void *dh, const void *b, const void *r,
                                                                      const float *rstd_post, const float *rstd_pre, const float *w_post,
                                                                      const float *gate, const float *w_pre, void *dx, void *db, float *dw_post,
                                                                      float *dgate, float *dw_pre, void *ws, size_t ws_bytes, void *stream)
{
    cudaStream_t st = (cudaStream_t)stream;
    int rc = check_join(d, "resnorm_bwd", b, gate, w_post, w_pre);
    if (rc) return rc;
    if ((db || dgate) && !b) return fail(QBP_ERR_INVALID_ARG, "resnorm_bwd: gradients of a block output that is NULL");
    if ((dw_post && !d->post) || (dw_pre && !d->pre)) return fail(QBP_ERR_INVALID_ARG, "resnorm_bwd: gradients of a norm that is not there");
    if (!dx && !db && !dw_post && !dgate && !dw_pre) return fail(QBP_ERR_INVALID_ARG, "resnorm_bwd: no output wanted");
    for (const float *w : {(const float *)dw_post, (const float *)dgate, (const float *)dw_pre, rstd_post, rstd_pre})
        if (!aligned_to(w, 4)) return fail(QBP_ERR_INVALID_ARG, "resnorm_bwd: misaligned fp32 tensors");
    const int64_t gates = gate || dgate ? join_gates(d) : 1;
    if (d->cols == 0) return QBP_OK;
    if (d->rows == 0) {
        if (dw_post) QBP_CUDA_OK(cudaMemsetAsync(dw_post, 0, (size_t)d->cols * 4, st));
        if (dw_pre) QBP_CUDA_OK(cudaMemsetAsync(dw_pre, 0, (size_t)d->cols * 4, st));
        if (dgate) QBP_CUDA_OK(cudaMemsetAsync(dgate, 0, (size_t)(gates * d->cols) * 4, st));
        return QBP_OK;
    }
    if ((dr && !real_ok(dr, d->x_dtype)) || (d->pre && (!real_ok(dh, d->b_dtype) || !real_ok(r, d->x_dtype) || !rstd_pre)) || (d->post && !rstd_post) ||
        (b && !real_ok(b, d->b_dtype)) || (dx && !real_ok(dx, d->x_dtype)) || (db && !real_ok(db, d->b_dtype)))
        return fail(QBP_ERR_INVALID_ARG, "resnorm_bwd: a tensor is NULL or misaligned");
    if (!dr && !d->pre) return fail(QBP_ERR_INVALID_ARG, "resnorm_bwd: neither output has a gradient");
    if (!ws || !aligned_to(ws, 256) || ws_bytes < qbp_resnorm_bwd_workspace_bytes(d))
        return fail(QBP_ERR_WORKSPACE, "resnorm_bwd: workspace NULL, misaligned or smaller than %zu bytes", qbp_resnorm_bwd_workspace_bytes(d));
    const bool per_gate = gate || dgate;
    const JoinCut c = join_cut(d, per_gate && d->gate_rows > 0);
    WsCarver w(ws, ws_bytes);
    JoinBwdParams P{};
    P.rows = d->rows; P.cols = d->cols; P.gate_rows = c.gate_rows; P.gates = c.gates; P.splits = c.splits; P.split_rows = c.split_rows;
    P.dr = dr; P.dh = dh; P.b = b; P.r = r; P.rstd_post = rstd_post; P.rstd_pre = rstd_pre; P.w_post = w_post; P.gate = gate; P.w_pre = w_pre;
    P.dx = dx; P.db = db; P.alpha = d->alpha; P.inv_cols = (float)(1.0 / (double)d->cols);
    P.post = d->post ? 1 : 0; P.pre = d->pre ? 1 : 0;
    P.part_post = w.take<float>((size_t)(c.blocks * d->cols)); P.part_pre = w.take<float>((size_t)(c.blocks * d->cols));
    P.part_gate = w.take<float>((size_t)(c.gates * c.splits * d->cols));
    P.sum_post = dw_post ? 1 : 0; P.sum_pre = dw_pre ? 1 : 0; P.sum_gate = dgate ? 1 : 0;
    if (dgate && c.splits == 1) P.part_gate = dgate;
    if (dw_post && c.blocks == 1) P.part_post = dw_post;
    if (dw_pre && c.blocks == 1) P.part_pre = dw_pre;
    const auto vec = [&](const void *p) { return aligned16(p); };
    P.vec_x = vec(dr) && vec(r) && vec(dx) && d->cols * (int64_t)dtype_size(d->x_dtype) % 16 == 0 ? 1 : 0;
    P.vec_b = vec(dh) && vec(b) && vec(db) && d->cols * (int64_t)dtype_size(d->b_dtype) % 16 == 0 ? 1 : 0;
    P.vec_w = vec(w_post) && vec(gate) && vec(w_pre) && d->cols % 4 == 0 ? 1 : 0;
    P.d = dropout_params(d->p, d->tensor_id, d->index_base);
    P.drop = P.d.threshold ? 1 : 0;
    const PhiloxKeys keys = philox_keys_host(d->seed);
    const JoinShape s = join_shape(d->cols);
    const size_t smem = s.warp ? (size_t)kJoinWarpRows * align_up((size_t)d->cols, 8) * 4 : 0;           // at most 32 KB
    QBP_TRACE_BEGIN(st);
    QBP_FOR_DTYPE(d->x_dtype, TX, QBP_FOR_DTYPE(d->b_dtype, TB, QBP_FOR_JOIN(s, CH, WARP, (launch(join_bwd_kernel<TX, TB, CH, WARP>, (unsigned)c.blocks, s.threads, smem, st, P, keys)))));
    QBP_LAUNCH_OK("join_bwd_kernel");
    JoinSums S{};
    int jobs = 0;
    int64_t outs = 1;
    if (dw_post && c.blocks > 1) S.j[jobs++] = {P.part_post, dw_post, 1, c.blocks};
    if (dw_pre && c.blocks > 1) S.j[jobs++] = {P.part_pre, dw_pre, 1, c.blocks};
    if (dgate && c.splits > 1) { S.j[jobs++] = {P.part_gate, dgate, c.gates, c.splits}; outs = c.gates; }
    if (!jobs) return QBP_OK;
    S.cols = d->cols;
    QBP_TRACE_BEGIN(st);
    launch(join_sum_kernel, dim3((unsigned)((d->cols + 31) / 32), (unsigned)std::min<int64_t>(outs, 1024), (unsigned)jobs), 32 * kSumHigh, 0, st, S);
    QBP_LAUNCH_OK("join_sum_kernel");
    return QBP_OK;
}

}  // namespace qbp
