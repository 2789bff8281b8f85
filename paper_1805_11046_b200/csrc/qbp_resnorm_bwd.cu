// Gradients of the join between two blocks (qbp_resnorm.cuh).
#include "qbp_resnorm.cuh"

namespace qbp {

struct JoinBwdParams {
    JoinItems it;
    const void *dr, *dh, *b, *r; const float *rstd_post, *rstd_pre, *w_post, *gate, *w_pre;
    void *dx, *db; float *part_post, *part_gate, *part_pre;
    float alpha, inv_cols;
    int post, pre, drop, x_dtype, b_dtype, slots, wide, sum_post, sum_gate, sum_pre;
    int *status;
    DropoutParams d;
};

// A thread's sums of one kind over an item's rows to the block's partial row, times parameters of its columns (nullable).  added: to
// what an item before of this block left there.  VEC: eight neighbouring columns, else 32 apart.
template <int CH, bool WARP, bool VEC>
__device__ __forceinline__ void join_leave(const float (&a)[CH][8], float *out, const float *w, int cols, int c0, int apart, bool added, float *fold, int threads)
{
    if (WARP) named_barrier(1, threads);
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        float m[8];
        load_params<VEC>(w, 0, c0 + k * apart, cols, m);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int c = c0 + k * apart + (VEC ? e : 32 * e);
            const float v = a[k][e] * m[e];
            if (WARP) fold[(threadIdx.x >> 5) * 256 * CH + c] = v;
            else if (c < cols) out[c] = added ? out[c] + v : v;
        }
    }
    if (WARP) {
        named_barrier(1, threads);
        for (int c = threadIdx.x; c < cols; c += threads) {
            float s = added ? out[c] : 0.0f;
#pragma unroll
            for (int q = 0; q < kJoinWarpRows; ++q) s += fold[q * 256 * CH + c];
            out[c] = s;
        }
    }
}

template <typename TX, typename TB, int CH, bool WARP, int MAXT, bool VEC>
__global__ void __launch_bounds__(MAXT, 1)
join_bwd_kernel(const __grid_constant__ JoinBwdParams P, const __grid_constant__ PhiloxKeys keys)
{
    constexpr bool kHold = CH == 1;                  // a row's values stay in registers behind the exchange, its slot is free with it
    extern __shared__ __align__(16) uint8_t ring[];
    __shared__ float fold[WARP ? kJoinWarpRows * 256 * CH : 1];            // WARP: the warps' sums
    __shared__ JoinScratch scratch;
    __shared__ JoinBars bars;
    const int lane = threadIdx.x & 31, all_warps = (int)(blockDim.x >> 5), warp = WARP ? 0 : threadIdx.x >> 5, warps = WARP ? 1 : all_warps;
    const int sub = WARP ? threadIdx.x >> 5 : 0, subs = WARP ? kJoinWarpRows : 1;
    const int cols = (int)P.it.cols, c0 = 256 * warp + (VEC ? 8 : 1) * lane, apart = 256 * warps;
    const uint32_t row_x = (uint32_t)cols * sizeof(TX), row_b = (uint32_t)cols * sizeof(TB);
    const uint32_t off_r = join_section<VEC>(row_x), off_h = 2u * off_r, off_b = off_h + join_section<VEC>(row_b), slot_bytes = off_b + join_section<VEC>(row_b);          // dr, r, dh, b
    join_bars_init(bars, all_warps);
    pdl_wait();
    if (blockIdx.x == 0 && threadIdx.x == 0) *P.status = 0;          // (a wait gives up a second later at the earliest)
    const uint32_t n_slots = kHold ? (uint32_t)P.slots : (uint32_t)kJoinBackSlots;
    uint8_t *const slots = ring + (uint32_t)sub * n_slots * slot_bytes;
    uint64_t *const full = bars.full[sub];
    const JoinSource src[4] = {{P.dr, row_x, 0u}, {P.pre ? P.r : nullptr, row_x, off_r}, {P.pre ? P.dh : nullptr, row_b, off_h}, {P.b, row_b, off_b}};
    bool dead = false;
    JoinPlace place{0u, 0u}, ahead{0u, 1u};          // of the row at hand, of the next row to be copied
    const auto fetch = [&](int64_t row) {
        if (WARP || warp == 0) {
            if (!WARP && !kHold) join_wait(&bars.empty[ahead.slot], ahead.ph, dead, P.status);
            if (!dead) join_copy<TX, TB, 2, VEC>(slots + ahead.slot * slot_bytes, &full[ahead.slot], src, row, P.it.rows);
            ahead = ahead.next(n_slots);
        }
    };
    In<VEC> in[CH];
    float gw[CH][8], w2[CH][8], a_pre[CH][8] = {};
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        in[k] = join_in<VEC>(c0 + k * apart, cols);
        join_gains<VEC>(P.w_pre, nullptr, 0, c0 + k * apart, cols, w2[k]);
    }
    const float factor = P.drop ? P.d.factor : 1.0f;
    int half = 0;
    for (int64_t item = blockIdx.x; item < P.it.gates * P.it.splits; item += gridDim.x) {
        const ItemRows rows = item_rows(P.it, item);
        float S[CH][8] = {};                          // of R dropout' b rstd_post
        float next1 = 1.0f, next2 = 0.0f;             // 1 / RMS of the next row, read a row ahead
        if (rows.first + sub < rows.end) {
            if (P.post) next1 = __ldg(P.rstd_post + rows.first + sub);
            if (P.pre) next2 = __ldg(P.rstd_pre + rows.first + sub);
        }
#pragma unroll
        for (int k = 0; k < CH; ++k) join_gains<VEC>(P.gate, P.post ? P.w_post : nullptr, rows.gate * cols, c0 + k * apart, cols, gw[k]);
        // (kHold: all slots are free, the last rows' sums have been exchanged)
        for (uint32_t k = 0; k < (kHold ? n_slots : 1u); ++k)
            if (rows.first + sub + (int64_t)k * subs < rows.end) fetch(rows.first + sub + (int64_t)k * subs);
        for (int64_t row = rows.first + sub; row < rows.end; row += subs) {
            const int64_t at = row * cols + c0;
            const float rstd1 = next1, rstd2 = next2;
            if (row + subs < rows.end) {
                if (P.post) next1 = __ldg(P.rstd_post + row + subs);
                if (P.pre) next2 = __ldg(P.rstd_pre + row + subs);
                if (!kHold) fetch(row + subs);
            }
            join_wait(&full[place.slot], place.ph, dead, P.status);
            const uint8_t *const slot = slots + place.slot * slot_bytes;
            const auto row_in = [&](int k) { return slot + src[k].offset + (VEC ? 0u : join_shift(src[k], row)); };
            const uint8_t *const my_g = row_in(0), *const my_r = row_in(1), *const my_h = row_in(2), *const my_b = row_in(3);
            const auto get_g = [&](int k, float (&v)[8]) { ring_read<TX, VEC>(my_g, c0 + k * apart, in[k] && P.dr, v); };
            const auto get_r = [&](int k, float (&v)[8]) { ring_read<TX, VEC>(my_r, c0 + k * apart, in[k] && P.pre, v); };
            const auto get_h = [&](int k, float (&v)[8]) { ring_read<TB, VEC>(my_h, c0 + k * apart, in[k] && P.pre, v); };
            const auto get_b = [&](int k, float (&v)[8]) { ring_read<TB, VEC>(my_b, c0 + k * apart, in[k] && P.b, v); };
            // Both means from one exchange: the second, of v w_post b, is linear in the first, m, with R = (dr + dh w_pre rstd_pre) - r m.
            float sums[3] = {0.0f, 0.0f, 0.0f};
            uint32_t kept = 0;                        // which elements the dropout keeps, a bit each
            float V[8], held_r[8], held_b[8];         // of eight columns: dr + dh w_pre rstd_pre, r, b
            {
#pragma unroll
                for (int k = 0; k < CH; ++k) {
                    float h[8], r[8], g[8], b[8];
                    get_h(k, h); get_r(k, r); get_g(k, g); get_b(k, b);
                    if (kHold) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) { held_r[e] = r[e]; held_b[e] = b[e]; }
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        a_pre[k][e] = fmaf(h[e] * r[e], rstd2, a_pre[k][e]);
                        h[e] *= w2[k][e];
                        sums[0] = fmaf(h[e], r[e], sums[0]);
                        b[e] *= gw[k][e];
                        g[e] = fmaf(h[e], rstd2, g[e]);
                        if (kHold) V[e] = g[e];
                    }
                    if (P.drop) {                     // (what is dropped has no part in the sums, whatever its gradient is: chosen, not multiplied by zero)
                        Kept<VEC> q;
                        q.make(P.d, keys, P.drop, at - (VEC ? 8 : 1) * lane + k * apart, 0);
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (q[e]) {               // (the sums: of use with a norm after the block alone)
                                kept |= 1u << (8 * k + e);
                                sums[1] = fmaf(g[e], b[e], sums[1]);
                                sums[2] = fmaf(r[e], b[e], sums[2]);
                            }
                    } else if (P.post) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            sums[1] = fmaf(g[e], b[e], sums[1]);
                            sums[2] = fmaf(r[e], b[e], sums[2]);
                        }
                    }
                }
            }
            if (kHold) __syncwarp();
            if (kHold || P.pre || P.post) { group_sums<WARP>(sums, scratch, half, warps); half ^= 1; }
            if (kHold && row + (int64_t)n_slots * subs < rows.end) fetch(row + (int64_t)n_slots * subs);
            // R = dr + rstd2 (dh w_pre) - r m2;  db = z rstd1 - b m1 with z = R dropout' gate w_post
            const float m2 = P.pre ? sums[0] * P.inv_cols * rstd2 * rstd2 * rstd2 : 0.0f;
            const float m1 = P.post ? (sums[1] - m2 * sums[2]) * factor * P.inv_cols * rstd1 * rstd1 * rstd1 : 0.0f;
            const float f1 = factor * rstd1;
            {
#pragma unroll
                for (int k = 0; k < CH; ++k) {
                    float R[8];
                    if (kHold) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) R[e] = fmaf(-held_r[e], m2, V[e]);
                    } else if (get_g(k, R); P.pre) {
                        float h[8], r[8];
                        get_h(k, h); get_r(k, r);
#pragma unroll
                        for (int e = 0; e < 8; ++e) R[e] = fmaf(-r[e], m2, fmaf(h[e] * w2[k][e], rstd2, R[e]));
                    }
                    if (P.b) {
                        float b[8], z[8];
                        if (kHold) {
#pragma unroll
                            for (int e = 0; e < 8; ++e) b[e] = held_b[e];
                        } else get_b(k, b);
#pragma unroll
                        for (int e = 0; e < 8; ++e) z[e] = R[e] * f1;
                        if (P.drop) {
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                const bool on = (kept >> (8 * k + e)) & 1u;
                                z[e] = on ? z[e] : 0.0f;
                                S[k][e] = on ? fmaf(z[e], b[e], S[k][e]) : S[k][e];
                            }
                        } else {
#pragma unroll
                            for (int e = 0; e < 8; ++e) S[k][e] = fmaf(z[e], b[e], S[k][e]);
                        }
                        if (P.db) {
#pragma unroll
                            for (int e = 0; e < 8; ++e) z[e] = P.post ? fmaf(-b[e], m1, z[e] * gw[k][e]) : z[e] * gw[k][e];
                            join_put<TB, VEC>(P.db, at + k * apart, in[k], P.wide, z);
                        }
                    }
                    if (P.dx) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) R[e] *= P.alpha;
                        join_put<TX, VEC>(P.dx, at + k * apart, in[k], P.wide, R);
                    }
                }
            }
            if (!kHold) {
                __syncwarp();
                if (!WARP && lane == 0) mbar_arrive(&bars.empty[place.slot]);
            }
            place = place.next(n_slots);
        }
        if (P.sum_gate) join_leave<CH, WARP, VEC>(S, P.part_gate + item * cols, P.post ? P.w_post : nullptr, cols, c0, apart, false, fold, 32 * all_warps);
        if (P.sum_post)
            join_leave<CH, WARP, VEC>(S, P.part_post + (int64_t)blockIdx.x * cols, P.gate ? P.gate + rows.gate * cols : nullptr, cols, c0, apart, item != blockIdx.x, fold, 32 * all_warps);
    }
    if (P.sum_pre) join_leave<CH, WARP, VEC>(a_pre, P.part_pre + (int64_t)blockIdx.x * cols, nullptr, cols, c0, apart, false, fold, 32 * all_warps);
}

template <typename TX, typename TB, int CH> struct JoinBwdRow { Held<TX> g[CH], r[CH]; Held<TB> h[CH], b[CH]; };

template <typename TX, typename TB, bool VEC>
__global__ void __launch_bounds__(512, 1)
join_bwd_wide_kernel(const __grid_constant__ JoinBwdParams P, const __grid_constant__ PhiloxKeys keys)
{
    constexpr int CH = kJoinWide;
    __shared__ JoinScratch scratch;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int cols = (int)P.it.cols;
    const auto w0 = [&](int k) { return 256 * (warp + k * warps); };
    const auto col = [&](int k) { return w0(k) + (VEC ? 8 * lane : lane); };
    const auto fetch = [&](JoinBwdRow<TX, TB, CH> &R, int64_t row) {
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            if (P.dr) load_row(R.g[k], P.dr, row * (int64_t)cols, col(k), cols, P.x_dtype);
            if (P.pre) { load_row(R.r[k], P.r, row * (int64_t)cols, col(k), cols, P.x_dtype); load_row(R.h[k], P.dh, row * (int64_t)cols, col(k), cols, P.b_dtype); }
            if (P.b) load_row(R.b[k], P.b, row * (int64_t)cols, col(k), cols, P.b_dtype);
        }
    };
    float a_pre[CH][8] = {};
    pdl_wait();
    if (blockIdx.x == 0 && threadIdx.x == 0) *P.status = 0;           // (nothing here waits)
    for (int64_t item = blockIdx.x; item < P.it.gates * P.it.splits; item += gridDim.x) {
        const ItemRows rows = item_rows(P.it, item);
        float S[CH][8] = {};
        JoinBwdRow<TX, TB, CH> R;
        for (int64_t row = rows.first; row < rows.end; ++row) {
            fetch(R, row);
            const int64_t base = row * (int64_t)cols;
            const float rstd1 = P.post ? __ldg(P.rstd_post + row) : 1.0f, rstd2 = P.pre ? __ldg(P.rstd_pre + row) : 0.0f;
            const auto get_g = [&](int k, float (&v)[8]) { unpack8(R.g[k], v); };
            const auto get_r = [&](int k, float (&v)[8]) { unpack8(R.r[k], v); };
            const auto get_h = [&](int k, float (&v)[8]) { unpack8(R.h[k], v); };
            const auto get_b = [&](int k, float (&v)[8]) { unpack8(R.b[k], v); };
            float mean2 = 0.0f;
            if (P.pre) {
                float s = 0.0f;
#pragma unroll
                for (int k = 0; k < CH; ++k) {
                    float h[8], r[8], w[8];
                    get_h(k, h); get_r(k, r);
                    load_params<VEC>(P.w_pre, 0, col(k), cols, w);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float t = h[e] * (r[e] * rstd2);
                        a_pre[k][e] += t;
                        s = fmaf(t, w[e], s);
                    }
                }
                mean2 = group_sum<false>(s, scratch, 0, warps) * P.inv_cols;
            }
            float s1 = 0.0f, z[CH][8];                   // z = R dropout' gate w_post
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                float g[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) g[e] = 0.0f;
                if (P.dr) get_g(k, g);
                if (P.pre) {
                    float h[8], r[8], w[8];
                    get_h(k, h); get_r(k, r);
                    load_params<VEC>(P.w_pre, 0, col(k), cols, w);
                    const float m = mean2 * rstd2;
#pragma unroll
                    for (int e = 0; e < 8; ++e) g[e] = fmaf(rstd2, h[e] * w[e] - r[e] * m, g[e]);
                }
                if (P.b) {
                    float b[8], w[8];
                    get_b(k, b);
                    Kept<VEC> kept;
                    if (P.drop) kept.make(P.d, keys, P.drop, base, w0(k));
                    const float f = P.drop ? P.d.factor : 1.0f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const bool keep = !P.drop || kept[e];
                        z[k][e] = keep ? g[e] * f : 0.0f;
                        b[e] *= rstd1;
                        S[k][e] = fmaf(z[k][e], keep ? b[e] : 0.0f, S[k][e]);
                    }
                    load_params<VEC>(P.gate, rows.gate * (int64_t)cols, col(k), cols, w);
#pragma unroll
                    for (int e = 0; e < 8; ++e) z[k][e] *= w[e];
                    if (P.post) {
                        load_params<VEC>(P.w_post, 0, col(k), cols, w);
#pragma unroll
                        for (int e = 0; e < 8; ++e) { z[k][e] *= w[e]; s1 = fmaf(z[k][e], b[e], s1); }
                    }
                }
                if (P.dx) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) g[e] *= P.alpha;
                    store_row(R.g[k], P.dx, base, col(k), cols, P.x_dtype, g);
                }
            }
            if (P.b) {
                const float mean1 = P.post ? group_sum<false>(s1, scratch, 1, warps) * P.inv_cols * rstd1 : 0.0f;
                if (P.db) {
#pragma unroll
                    for (int k = 0; k < CH; ++k) {
                        if (P.post) {
                            float b[8];
                            get_b(k, b);
#pragma unroll
                            for (int e = 0; e < 8; ++e) z[k][e] = rstd1 * (z[k][e] - b[e] * mean1);
                        }
                        store_row(R.b[k], P.db, base, col(k), cols, P.b_dtype, z[k]);
                    }
                }
            }
            if (P.pre != P.post) __syncthreads();            // (the next row's sum goes where this one's is still read from)
        }
        if (P.sum_gate) join_leave<CH, false, VEC>(S, P.part_gate + item * (int64_t)cols, P.post ? P.w_post : nullptr, cols, col(0), 256 * warps, false, nullptr, (int)blockDim.x);
        if (P.sum_post)
            join_leave<CH, false, VEC>(S, P.part_post + (int64_t)blockIdx.x * cols, P.gate ? P.gate + rows.gate * (int64_t)cols : nullptr, cols, col(0), 256 * warps,
                                      item != blockIdx.x, nullptr, (int)blockDim.x);
    }
    if (P.sum_pre) join_leave<CH, false, VEC>(a_pre, P.part_pre + (int64_t)blockIdx.x * cols, nullptr, cols, col(0), 256 * warps, false, nullptr, (int)blockDim.x);
}

// out[o][c] = sum over `count` partial rows in [outs][count][cols], in a fixed order: the thirty-two warps of a block take every
// thirty-second row, 32 V columns of it, eight loads at a time (a sum waits for its loads and for nothing else), then the thirty-two are
// added up.  V: 4 where rows are whole groups of four floats (147 rows of 4096, twice: 7.7 to 8.7 us; of
// 293 rows, three times, 11.1 us and with one column a lane 14.7).
struct JoinSum { const float *part; float *out; int64_t outs, count; };
struct JoinSums { JoinSum j[3]; int64_t cols; };
constexpr int kSumHigh = 32, kSumAhead = 8;
template <int V> struct Floats { float v[V]; };
template <int V>
__global__ void __launch_bounds__(32 * kSumHigh) join_sum_kernel(const __grid_constant__ JoinSums S)
{
    using F = Floats<V>;
    __shared__ __align__(16) F s_part[kSumHigh][33];
    const JoinSum &j = S.j[blockIdx.z];
    const int lane = threadIdx.x & 31, high = threadIdx.x >> 5;
    const int64_t c0 = (int64_t)blockIdx.x * 32 * V, c = c0 + lane * V;
    const auto load = [](const float *p) {
        F f;
        if constexpr (V == 4) *reinterpret_cast<float4 *>(f.v) = *reinterpret_cast<const float4 *>(p);
        else f.v[0] = *p;
        return f;
    };
    pdl_wait();
    for (int64_t o = blockIdx.y; o < j.outs; o += gridDim.y) {
        F s = {};
        if (c < S.cols) {
            const float *p = j.part + o * j.count * S.cols + c;
            for (int64_t k = high; k < j.count; k += kSumHigh * kSumAhead) {
                F v[kSumAhead];
#pragma unroll
                for (int a = 0; a < kSumAhead; ++a) v[a] = k + a * kSumHigh < j.count ? load(p + (k + a * kSumHigh) * S.cols) : F{};
#pragma unroll
                for (int a = 0; a < kSumAhead; ++a)
#pragma unroll
                    for (int e = 0; e < V; ++e) s.v[e] += v[a].v[e];
            }
        }
        s_part[high][lane] = s;
        __syncthreads();
        // each warp adds up V columns
        s = s_part[lane][high];
#pragma unroll
        for (int q = 16; q > 0; q >>= 1)
#pragma unroll
            for (int e = 0; e < V; ++e) s.v[e] += __shfl_xor_sync(0xFFFFFFFFu, s.v[e], q);
        if (lane == 0) {
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (c0 + high * V + e < S.cols) j.out[o * S.cols + c0 + high * V + e] = s.v[e];
        }
        __syncthreads();
    }
}

// ================================================================= host side
// Partial rows of dgate: none where an item is all of a gate's rows, whose sum is the gradient.
static size_t gate_parts(const JoinItems &it) { return it.splits > 1 ? (size_t)(it.gates * it.splits * it.cols) : 0; }
static JoinCut join_cut_bwd(const qbp_resnorm_desc *d, const JoinShape &s, bool per_gate)
{
    return join_cut(d, s, per_gate, join_blocks(d, s, 2), s.warp ? 2 : 4, true);
}

extern "C" __attribute__((visibility("default"))) size_t qbp_resnorm_bwd_workspace_bytes(const qbp_resnorm_desc *d)
{
    if (!d || !join_extents_ok(d) || d->rows == 0 || d->cols == 0) return 256;
    size_t most = 0;
    // (with and without a gate, rows on the 16-byte boundaries and off them, as far as these are cut differently)
    const JoinShape off = join_shape(d, 2, false), on = join_shape(d, 2, true);
    const bool gates = join_gate_rows(d) < d->rows, both = d->cols % 8 == 0 && (on.ch != off.ch || join_blocks(d, on, 2) != join_blocks(d, off, 2));
    for (int k = 0; k < 4; ++k) {
        if (((k & 1) && !gates) || ((k & 2) && !both)) continue;
        const JoinCut c = join_cut_bwd(d, k & 2 ? on : off, (k & 1) != 0);
        most = std::max(most, 2 * align_up((size_t)(c.blocks * d->cols) * 4, 256) + align_up(gate_parts(c.it) * 4, 256));
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
    for (const float *w : {(const float *)dw_post, (const float *)dgate, (const float *)dw_pre, rstd_post, rstd_pre})
        if (!aligned_to(w, 4)) return fail(QBP_ERR_INVALID_ARG, "resnorm_bwd: misaligned fp32 tensors");
    if ((dw_post && !d->post) || (dw_pre && !d->pre)) return fail(QBP_ERR_INVALID_ARG, "resnorm_bwd: gradients of a norm that is not there");
    if (d->cols == 0) return join_empty(ws, ws_bytes, st);
    if (d->rows == 0) {                              // (no gates but for one that all rows share)
        if (dw_post) QBP_CUDA_OK(cudaMemsetAsync(dw_post, 0, (size_t)d->cols * 4, st));
        if (dw_pre) QBP_CUDA_OK(cudaMemsetAsync(dw_pre, 0, (size_t)d->cols * 4, st));
        if (dgate && !d->gate_rows) QBP_CUDA_OK(cudaMemsetAsync(dgate, 0, (size_t)d->cols * 4, st));
        return join_empty(ws, ws_bytes, st);
    }
    if ((db || dgate) && !b) return fail(QBP_ERR_INVALID_ARG, "resnorm_bwd: gradients of a block output that is NULL");
    if (!dx && !db && !dw_post && !dgate && !dw_pre) return fail(QBP_ERR_INVALID_ARG, "resnorm_bwd: no output wanted");
    if ((dr && !real_ok(dr, d->x_dtype)) || (d->pre && (!real_ok(dh, d->b_dtype) || !real_ok(r, d->x_dtype) || !rstd_pre)) || (d->post && !rstd_post) ||
        (b && !real_ok(b, d->b_dtype)) || (dx && !real_ok(dx, d->x_dtype)) || (db && !real_ok(db, d->b_dtype)))
        return fail(QBP_ERR_INVALID_ARG, "resnorm_bwd: a tensor is NULL or misaligned");
    if (!dr && !d->pre) return fail(QBP_ERR_INVALID_ARG, "resnorm_bwd: neither output has a gradient");
    if (!ws || !aligned_to(ws, 256) || ws_bytes < qbp_resnorm_bwd_workspace_bytes(d))
        return fail(QBP_ERR_WORKSPACE, "resnorm_bwd: workspace NULL, misaligned or smaller than %zu bytes", qbp_resnorm_bwd_workspace_bytes(d));
    const bool vec = d->cols % 8 == 0 && aligned16(dr) && aligned16(dh) && aligned16(b) && aligned16(r) && aligned16(dx) && aligned16(db) && aligned16(w_post) &&
                     aligned16(gate) && aligned16(w_pre);
    const JoinShape s = join_shape(d, 2, vec);
    const JoinCut c = join_cut_bwd(d, s, gate || dgate);
    WsCarver w(ws, ws_bytes);
    JoinBwdParams P{};
    P.status = w.take<int>(1);
    P.it = c.it;
    P.dr = dr; P.dh = dh; P.b = b; P.r = r; P.rstd_post = rstd_post; P.rstd_pre = rstd_pre; P.w_post = w_post; P.gate = gate; P.w_pre = w_pre;
    P.dx = dx; P.db = db; P.alpha = d->alpha; P.inv_cols = (float)(1.0 / (double)d->cols);
    P.post = d->post ? 1 : 0; P.pre = d->pre ? 1 : 0; P.x_dtype = d->x_dtype; P.b_dtype = d->b_dtype;
    P.part_post = w.take<float>((size_t)(c.blocks * d->cols)); P.part_pre = w.take<float>((size_t)(c.blocks * d->cols));
    P.sum_post = dw_post ? 1 : 0; P.sum_pre = dw_pre ? 1 : 0; P.sum_gate = dgate ? 1 : 0;
    P.part_gate = c.it.splits > 1 ? w.take<float>(gate_parts(c.it)) : dgate;
    if (dw_post && c.blocks == 1) P.part_post = dw_post;
    if (dw_pre && c.blocks == 1) P.part_pre = dw_pre;
    P.d = dropout_params(d->p, d->tensor_id, d->index_base);
    P.drop = P.d.threshold == 65536u ? 2 : P.d.threshold ? 1 : 0;
    P.slots = join_slots(d, s, 2);
    P.wide = aligned_to(dx, 32) && aligned_to(db, 32) ? 1 : 0;
    const PhiloxKeys keys = philox_keys_host(d->seed);
    QBP_TRACE_BEGIN(st);
    if (s.ch <= 2)
        QBP_FOR_DTYPE(d->x_dtype, TX, QBP_FOR_DTYPE(d->b_dtype, TB, QBP_FOR_JOIN(s, true, CH, WARP, MAXT, {
            static PerDeviceOnce once[2];
            if ((rc = launch_join(vec ? join_bwd_kernel<TX, TB, CH, WARP, MAXT, true> : join_bwd_kernel<TX, TB, CH, WARP, MAXT, false>, once[vec], c.blocks, s, join_ring(d, s, 2), st, P, keys))) return rc;
        })));
    else if (vec)
        QBP_FOR_DTYPE(d->x_dtype, TX, QBP_FOR_DTYPE(d->b_dtype, TB, (launch(join_bwd_wide_kernel<TX, TB, true>, dim3((unsigned)c.blocks), s.threads, 0, st, P, keys))));
    else
        launch(join_bwd_wide_kernel<AnyReal, AnyReal, false>, dim3((unsigned)c.blocks), s.threads, 0, st, P, keys);
    QBP_LAUNCH_OK("join_bwd_kernel");
    JoinSums S{};
    int jobs = 0;
    int64_t outs = 1;
    if (dw_post && c.blocks > 1) S.j[jobs++] = {P.part_post, dw_post, 1, c.blocks};
    if (dw_pre && c.blocks > 1) S.j[jobs++] = {P.part_pre, dw_pre, 1, c.blocks};
    if (dgate && c.it.splits > 1) { S.j[jobs++] = {P.part_gate, dgate, c.it.gates, c.it.splits}; outs = c.it.gates; }
    if (!jobs) return QBP_OK;
    S.cols = d->cols;
    // (the parts are in the workspace, on 256-byte boundaries)
    const dim3 grid((unsigned)((d->cols + (d->cols % 4 ? 31 : 127)) / (d->cols % 4 ? 32 : 128)), (unsigned)std::min<int64_t>(outs, 1024), (unsigned)jobs);
    QBP_TRACE_BEGIN(st);
    if (d->cols % 4 == 0) launch(join_sum_kernel<4>, grid, 32 * kSumHigh, 0, st, S);
    else                  launch(join_sum_kernel<1>, grid, 32 * kSumHigh, 0, st, S);
    QBP_LAUNCH_OK("join_sum_kernel");
    return QBP_OK;
}

}  // namespace qbp
