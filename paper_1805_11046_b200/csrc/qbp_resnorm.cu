// Forward of the join between two blocks (qbp_resnorm.cuh).
#include "qbp_resnorm.cuh"

namespace qbp {

struct JoinParams {
    JoinItems it;
    const void *x, *b; const float *w_post, *gate, *w_pre;
    void *r, *h; float *rstd_post, *rstd_pre;
    float eps, alpha, inv_cols;
    int post, pre, drop, x_dtype, b_dtype, slots, wide;      // wide: outputs of fp32 start on 32-byte boundaries
    int *status;
    DropoutParams d;
};

template <typename TX, typename TB, int CH, bool WARP, int MAXT, bool VEC>
__global__ void __launch_bounds__(MAXT, MAXT == 256 ? 2 : 1)
join_fwd_kernel(const __grid_constant__ JoinParams P, const __grid_constant__ PhiloxKeys keys)
{
    extern __shared__ __align__(16) uint8_t ring[];
    __shared__ JoinScratch scratch;
    __shared__ JoinBars bars;
    const int lane = threadIdx.x & 31, all_warps = (int)(blockDim.x >> 5), warp = WARP ? 0 : threadIdx.x >> 5, warps = WARP ? 1 : all_warps;
    const int sub = WARP ? threadIdx.x >> 5 : 0, subs = WARP ? kJoinWarpRows : 1;
    const int cols = (int)P.it.cols, c0 = 256 * warp + (VEC ? 8 : 1) * lane, apart = 256 * warps;      // the thread's first column, and its next ones'
    const uint32_t row_x = (uint32_t)cols * sizeof(TX), row_b = (uint32_t)cols * sizeof(TB), off_b = join_section<VEC>(row_x), slot_bytes = off_b + join_section<VEC>(row_b);
    join_bars_init(bars, all_warps);
    pdl_wait();
    if (blockIdx.x == 0 && threadIdx.x == 0) *P.status = 0;          // (a wait gives up a second later at the earliest)
    const uint32_t n_slots = (uint32_t)P.slots;
    uint8_t *const slots = ring + (uint32_t)sub * n_slots * slot_bytes;
    uint64_t *const full = bars.full[sub];
    const JoinSource src[2] = {{P.x, row_x, 0u}, {P.b, row_b, off_b}};
    bool dead = false;
    const auto fetch = [&](int64_t row, int64_t end, uint32_t slot) {
        if ((WARP || warp == 0) && row < end && !dead) join_copy<TX, TB, 1, VEC>(slots + slot * slot_bytes, &full[slot], src, row, P.it.rows);
    };
    In<VEC> in[CH];
    float gw[CH][8], w2[CH][8];
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        in[k] = join_in<VEC>(c0 + k * apart, cols);
        join_gains<VEC>(P.w_pre, nullptr, 0, c0 + k * apart, cols, w2[k]);
    }
    const auto x_in = [&](uint32_t slot, int64_t row) { return slots + slot * slot_bytes + (VEC ? 0u : join_shift(src[0], row)); };
    const auto b_in = [&](uint32_t slot, int64_t row) { return slots + slot * slot_bytes + off_b + (VEC ? 0u : join_shift(src[1], row)); };
    const auto square_sum = [&](uint32_t slot, int64_t row) {
        const uint8_t *const my_b = b_in(slot, row);
        float s = 0.0f;
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            float v[8];
            ring_read<TB, VEC>(my_b, c0 + k * apart, in[k], v);
#pragma unroll
            for (int e = 0; e < 8; ++e) s = fmaf(v[e], v[e], s);
        }
        return s;
    };
    const float factor = P.drop ? P.d.factor : 1.0f;
    int64_t had = -1;
    int half = 0;
    JoinPlace place{0u, 0u};
    for (int64_t item = blockIdx.x; item < P.it.gates * P.it.splits; item += gridDim.x) {
        const ItemRows rows = item_rows(P.it, item);
        if (P.b && rows.gate != had) {
#pragma unroll
            for (int k = 0; k < CH; ++k) join_gains<VEC>(P.gate, P.post ? P.w_post : nullptr, rows.gate * cols, c0 + k * apart, cols, gw[k]);
            had = rows.gate;
        }
        // (all slots are free: the last rows' sums have been exchanged)
        JoinPlace p = place;
        for (uint32_t k = 0; k < n_slots; ++k) { fetch(rows.first + sub + k * subs, rows.end, p.slot); p = p.next(n_slots); }
        float rstd = 1.0f;
        if (rows.first + sub < rows.end) {
            join_wait(&full[place.slot], place.ph, dead, P.status);
            if (P.post) { rstd = rsqrtf(group_sum<WARP>(square_sum(place.slot, rows.first + sub), scratch, half, warps) * P.inv_cols + P.eps); half ^= 1; }
        }
        for (int64_t row = rows.first + sub; row < rows.end; row += subs) {
            const int64_t at = row * cols + c0;
            const float scale = factor * rstd;
            float r[CH][8], sums[2] = {0.0f, 0.0f};           // of this row's r^2, of the next row's b^2
            if (P.post && P.rstd_post && warp == 0 && lane == 0) P.rstd_post[row] = rstd;
            {
                const uint8_t *const my_x = x_in(place.slot, row), *const my_b = b_in(place.slot, row);
#pragma unroll
                for (int k = 0; k < CH; ++k) {
                    ring_read<TX, VEC>(my_x, c0 + k * apart, in[k], r[k]);
#pragma unroll
                    for (int e = 0; e < 8; ++e) r[k][e] *= P.alpha;
                    if (P.b) {
                        float b[8];
                        ring_read<TB, VEC>(my_b, c0 + k * apart, in[k], b);
if (P.drop) {                 // (what is dropped counts for nothing, whatever it or its row's norm is: chosen, not multiplied by zero)
                            Kept<VEC> kept;
                            kept.make(P.d, keys, P.drop, row * cols, 256 * warp + k * apart);
#pragma unroll
                            for (int e = 0; e < 8; ++e) b[e] = kept[e] ? b[e] * scale : 0.0f;
                        } else {
#pragma unroll
                            for (int e = 0; e < 8; ++e) b[e] *= scale;
                        }
#pragma unroll
                        for (int e = 0; e < 8; ++e) r[k][e] = fmaf(b[e], gw[k][e], r[k][e]);
                    }
                    join_put<TX, VEC>(P.r, at + k * apart, in[k], P.wide, r[k]);
#pragma unroll
                    for (int e = 0; e < 8; ++e) sums[0] = fmaf(r[k][e], r[k][e], sums[0]);    // (zero behind the last column, as x and b are)
                }
            }
            const JoinPlace following = place.next(n_slots);
            if (row + subs < rows.end) {
                join_wait(&full[following.slot], following.ph, dead, P.status);
                if (P.post) sums[1] = square_sum(following.slot, row + subs);
            }
            __syncwarp();
            group_sums<WARP>(sums, scratch, half, warps);
            half ^= 1;
            fetch(row + (int64_t)n_slots * subs, rows.end, place.slot);
            place = following;
            rstd = P.post ? rsqrtf(sums[1] * P.inv_cols + P.eps) : 1.0f;
            if (P.pre) {
                const float rstd2 = rsqrtf(sums[0] * P.inv_cols + P.eps);
                if (P.rstd_pre && warp == 0 && lane == 0) P.rstd_pre[row] = rstd2;
#pragma unroll
                for (int k = 0; k < CH; ++k) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) r[k][e] = r[k][e] * rstd2 * w2[k][e];
                    join_put<TB, VEC>(P.h, at + k * apart, in[k], P.wide, r[k]);
                }
            }
        }
    }
}

template <typename TX, typename TB, int CH> struct JoinRow { Held<TX> x[CH]; Held<TB> b[CH]; };

template <typename TX, typename TB, bool VEC>
__global__ void __launch_bounds__(512, 1)
join_fwd_wide_kernel(const __grid_constant__ JoinParams P, const __grid_constant__ PhiloxKeys keys)
{
    constexpr int CH = kJoinWide;
    __shared__ JoinScratch scratch;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int cols = (int)P.it.cols;
    const auto w0 = [&](int k) { return 256 * (warp + k * warps); };
    const auto col = [&](int k) { return w0(k) + (VEC ? 8 * lane : lane); };
    const auto fetch = [&](JoinRow<TX, TB, CH> &R, int64_t row) {
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            load_row(R.x[k], P.x, row * (int64_t)cols, col(k), cols, P.x_dtype);
            if (P.b) load_row(R.b[k], P.b, row * (int64_t)cols, col(k), cols, P.b_dtype);
        }
    };
    pdl_wait();
    if (blockIdx.x == 0 && threadIdx.x == 0) *P.status = 0;           // (nothing here waits)
    for (int64_t item = blockIdx.x; item < P.it.gates * P.it.splits; item += gridDim.x) {
        const ItemRows rows = item_rows(P.it, item);
        JoinRow<TX, TB, CH> R;
        for (int64_t row = rows.first; row < rows.end; ++row) {
            fetch(R, row);
            const int64_t base = row * (int64_t)cols;
            const auto get_x = [&](int k, float (&v)[8]) { unpack8(R.x[k], v); };
            const auto get_b = [&](int k, float (&v)[8]) { unpack8(R.b[k], v); };
            float rstd = 1.0f;
            if (P.post) {
                float s = 0.0f;
#pragma unroll
                for (int k = 0; k < CH; ++k) {
                    float v[8];
                    get_b(k, v);
#pragma unroll
                    for (int e = 0; e < 8; ++e) s = fmaf(v[e], v[e], s);
                }
                rstd = rsqrtf(group_sum<false>(s, scratch, 0, warps) * P.inv_cols + P.eps);
                if (P.rstd_post && warp == 0 && lane == 0) P.rstd_post[row] = rstd;
            }
            float s2 = 0.0f, r8[CH][8];
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                get_x(k, r8[k]);
#pragma unroll
                for (int e = 0; e < 8; ++e) r8[k][e] *= P.alpha;
                if (P.b) {
                    float b[8], w[8];
                    get_b(k, b);
                    const float scale = P.drop ? rstd * P.d.factor : rstd;
#pragma unroll
                    for (int e = 0; e < 8; ++e) b[e] *= scale;
                    if (P.post && P.w_post) {
                        load_params<VEC>(P.w_post, 0, col(k), cols, w);
#pragma unroll
                        for (int e = 0; e < 8; ++e) b[e] *= w[e];
                    }
                    load_params<VEC>(P.gate, rows.gate * (int64_t)cols, col(k), cols, w);
                    Kept<VEC> kept;
                    if (P.drop) kept.make(P.d, keys, P.drop, base, w0(k));
                    // (what is dropped counts for nothing, whatever it is: chosen, not multiplied by zero)
#pragma unroll
                    for (int e = 0; e < 8; ++e) b[e] = !P.drop || kept[e] ? b[e] : 0.0f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) r8[k][e] = fmaf(b[e], w[e], r8[k][e]);
                }
                store_row(R.x[k], P.r, base, col(k), cols, P.x_dtype, r8[k]);
#pragma unroll
                for (int e = 0; e < 8; ++e) s2 = fmaf(r8[k][e], r8[k][e], s2);      // (zero behind the last column, as x and b are)
            }
            if (P.pre) {
                const float rstd2 = rsqrtf(group_sum<false>(s2, scratch, 1, warps) * P.inv_cols + P.eps);
                if (P.rstd_pre && warp == 0 && lane == 0) P.rstd_pre[row] = rstd2;
#pragma unroll
                for (int k = 0; k < CH; ++k) {
                    float w[8];
                    load_params<VEC>(P.w_pre, 0, col(k), cols, w);
#pragma unroll
                    for (int e = 0; e < 8; ++e) r8[k][e] = r8[k][e] * rstd2 * w[e];
                    store_row(R.b[k], P.h, base, col(k), cols, P.b_dtype, r8[k]);
                }
            }
            if (P.pre != P.post) __syncthreads();            // (the next row's sum goes where this one's is still read from)
        }
    }
}

extern "C" __attribute__((visibility("default"))) int qbp_resnorm_fwd(const qbp_resnorm_desc *d, const void *x, const void *b, const float *w_post,
                                                                      const float *gate, const float *w_pre, void *r, void *h, float *rstd_post,
                                                                      float *rstd_pre, void *ws, size_t ws_bytes, void *stream)
{
    cudaStream_t st = (cudaStream_t)stream;
    int rc = check_join(d, "resnorm_fwd", b, gate, w_post, w_pre);
    if (rc) return rc;
    if (d->rows == 0 || d->cols == 0) return join_empty(ws, ws_bytes, st);
    if (!real_ok(x, d->x_dtype) || (b && !real_ok(b, d->b_dtype)) || (r && !real_ok(r, d->x_dtype)) || (d->pre && !real_ok(h, d->b_dtype)))
        return fail(QBP_ERR_INVALID_ARG, "resnorm_fwd: a tensor is NULL or misaligned");
    if (!aligned_to(rstd_post, 4) || !aligned_to(rstd_pre, 4)) return fail(QBP_ERR_INVALID_ARG, "resnorm_fwd: misaligned fp32 tensors");
    if (!r && (b || d->alpha != 1.0f)) return fail(QBP_ERR_INVALID_ARG, "resnorm_fwd: r may be NULL only where it is x");
    if (!r && !d->pre) return fail(QBP_ERR_INVALID_ARG, "resnorm_fwd: no output wanted");
    if (!ws || !aligned_to(ws, 256) || ws_bytes < 256) return fail(QBP_ERR_WORKSPACE, "resnorm_fwd: workspace NULL, misaligned or smaller than 256 bytes");
    JoinParams P{};
    const bool vec = d->cols % 8 == 0 && aligned16(x) && aligned16(b) && aligned16(r) && aligned16(h) && aligned16(w_post) && aligned16(gate) && aligned16(w_pre);
    const JoinShape s = join_shape(d, 1, vec);
    const JoinCut c = join_cut(d, s, gate != nullptr, join_blocks(d, s, 1), 1, false);
    P.it = c.it;
    P.x = x; P.b = b; P.w_post = w_post; P.gate = gate; P.w_pre = w_pre; P.r = r; P.h = h; P.rstd_post = rstd_post; P.rstd_pre = rstd_pre;
    P.eps = d->eps; P.alpha = d->alpha; P.inv_cols = (float)(1.0 / (double)d->cols);
    P.post = d->post ? 1 : 0; P.pre = d->pre ? 1 : 0; P.x_dtype = d->x_dtype; P.b_dtype = d->b_dtype;
    P.d = dropout_params(d->p, d->tensor_id, d->index_base);
    P.drop = P.d.threshold == 65536u ? 2 : P.d.threshold ? 1 : 0;
    P.status = static_cast<int *>(ws);
    P.slots = join_slots(d, s, 1);
    P.wide = aligned_to(r, 32) && aligned_to(h, 32) ? 1 : 0;
    const PhiloxKeys keys = philox_keys_host(d->seed);
    QBP_TRACE_BEGIN(st);
    if (s.ch <= 2)
        QBP_FOR_DTYPE(d->x_dtype, TX, QBP_FOR_DTYPE(d->b_dtype, TB, QBP_FOR_JOIN(s, false, CH, WARP, MAXT, {
            static PerDeviceOnce once[2];
            if ((rc = launch_join(vec ? join_fwd_kernel<TX, TB, CH, WARP, MAXT, true> : join_fwd_kernel<TX, TB, CH, WARP, MAXT, false>, once[vec], c.blocks, s, join_ring(d, s, 1), st, P, keys))) return rc;
        })));
    else if (vec)
        QBP_FOR_DTYPE(d->x_dtype, TX, QBP_FOR_DTYPE(d->b_dtype, TB, (launch(join_fwd_wide_kernel<TX, TB, true>, dim3((unsigned)c.blocks), s.threads, 0, st, P, keys))));
    else
        launch(join_fwd_wide_kernel<AnyReal, AnyReal, false>, dim3((unsigned)c.blocks), s.threads, 0, st, P, keys);
    QBP_LAUNCH_OK("join_fwd_kernel");
    return QBP_OK;
}

}  // namespace qbp
