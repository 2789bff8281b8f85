// The join between two blocks of a residual network and its gradients (qbp_resnorm_fwd / _bwd in include/qbp.h): norm after a
// block, gate, dropout, residual stream and the norm before the next block, in one pass over the rows.
//
// A row is held in registers by the threads of one group: a warp (of a block's eight) for rows of up to 512 columns, a block of
// up to 512 threads beyond; a thread has CH times eight columns.  The two sums over a row (of b^2 and of r^2; backwards of the
// gradients' projections on r and b) are exchanged between the group's threads, forward a row's second with the next row's first, backwards
// both at once, and nothing is read twice.  A block
// takes neighbouring rows of one gate (an item) and keeps the parameters of its columns in registers.  Rows come through a ring of two
// or three in shared memory, copied whole by one thread (cp.async.bulk): a row is on its way while the one before is worked on, and stays
// out of the threads' registers.  (Copied by the threads that read it, 16 bytes each, a row of 48 KB took 2100 cycles of their time, of 5900.)
//
// Backwards, with gate and w_post constant along an item's columns, dw_post and dgate are multiples of one sum over its rows,
// S = sum of R dropout'(b rstd_post): dgate = w_post S, dw_post = gate S.  A thread keeps S and dw_pre's sum in registers, a block leaves
// one partial row of each, and a second kernel adds these up in a fixed order.
//
// Columns.  Rows whose tensors all start on 16-byte boundaries are read eight neighbouring columns to a thread (VEC); others
// with the lanes of a warp side by side, element by element, in a form for any type.
#include "qbp_dropout.cuh"

#include <algorithm>

namespace qbp {

constexpr int kJoinWarpRows = 8;                    // rows of a block whose groups are warps
constexpr int64_t kJoinMaxCols = QBP_RESNORM_MAX_COLS;

// How the rows are cut: `gates` gates of `gate_rows` rows, each in `splits` items of `split_rows` rows (the last one fewer).
struct JoinItems { int64_t rows, cols, gate_rows, gates, splits, split_rows; };

struct JoinParams {
    JoinItems it;
    const void *x, *b; const float *w_post, *gate, *w_pre;
    void *r, *h; float *rstd_post, *rstd_pre;
    float eps, alpha, inv_cols;
    int post, pre, drop, x_dtype, b_dtype, wide;      // wide: outputs of fp32 start on 32-byte boundaries
    int *status;
    DropoutParams d;
};

struct JoinBwdParams {
    JoinItems it;
    const void *dr, *dh, *b, *r; const float *rstd_post, *rstd_pre, *w_post, *gate, *w_pre;
    void *dx, *db; float *part_post, *part_gate, *part_pre;
    float alpha, inv_cols;
    int post, pre, drop, x_dtype, b_dtype, wide, sum_post, sum_gate, sum_pre;
    int *status;
    DropoutParams d;
};

#ifdef __CUDACC__
// Eight elements of a row as a thread holds them.  VEC: neighbours, as they lie in memory; else 32 columns apart, as floats.
struct AnyReal {};
template <typename T> struct Held { Raw8<T> raw; };
template <> struct Held<AnyReal> { float v[8]; };

template <typename T> __device__ __forceinline__ void unpack8(const Held<T> &h, float (&v)[8]) { unpack8(h.raw, v); }
__device__ __forceinline__ void unpack8(const Held<AnyReal> &h, float (&v)[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = h.v[e];
}
// c: the thread's first column; columns at and behind `cols` are zero.
template <typename T> __device__ __forceinline__ void load_row(Held<T> &h, const void *row0, int64_t base, int c, int cols, int)
{
    const T *p = static_cast<const T *>(row0) + base + c;
    const bool in = c < cols;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 2); ++i) h.raw.w[i] = in ? reinterpret_cast<const uint4 *>(p)[i] : make_uint4(0, 0, 0, 0);   // (not __ldg: an output may lie over an input)
}
template <typename T> __device__ __forceinline__ void load_strided(float (&v)[8], const void *row0, int64_t base, int c, int cols)
{
    const T *p = static_cast<const T *>(row0) + base + c;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = c + 32 * e < cols ? real_of(p[32 * e]) : 0.0f;
}
__device__ __forceinline__ void load_row(Held<AnyReal> &h, const void *row0, int64_t base, int c, int cols, int dtype)
{
    QBP_FOR_DTYPE(dtype, T, load_strided<T>(h.v, row0, base, c, cols));
}
// Rounds to the type and stores; v is what the stored values stand for.
template <typename T> __device__ __forceinline__ void store_row(const Held<T> &, void *row0, int64_t base, int c, int cols, int, float (&v)[8])
{
    const Raw8<T> r = pack8<T>(v);
    T *p = static_cast<T *>(row0) + base + c;
    if (row0 && c < cols) {
#pragma unroll
        for (int i = 0; i < (int)(sizeof(T) / 2); ++i) reinterpret_cast<uint4 *>(p)[i] = r.w[i];
    }
    unpack8(r, v);
}
template <typename T> __device__ __forceinline__ void store_strided(void *row0, int64_t base, int c, int cols, float (&v)[8])
{
    T *p = static_cast<T *>(row0) + base + c;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const T t = real_to<T>(v[e]);
        if (row0 && c + 32 * e < cols) p[32 * e] = t;
        v[e] = real_of(t);
    }
}
__device__ __forceinline__ void store_row(const Held<AnyReal> &, void *row0, int64_t base, int c, int cols, int dtype, float (&v)[8])
{
    QBP_FOR_DTYPE(dtype, T, store_strided<T>(row0, base, c, cols, v));
}
// fp32 parameters of the thread's columns (absent: ones; behind the last column anything).
template <bool VEC> __device__ __forceinline__ void load_params(const float *p, int64_t base, int c, int cols, float (&v)[8])
{
    if (!p) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = 1.0f;
    } else if (VEC) {
        Held<float> h;
        load_row(h, p, base, c, cols, QBP_F32);
        unpack8(h, v);
    } else {
        load_strided<float>(v, p, base, c, cols);
    }
}
// Which of a thread's eight elements a dropout keeps.  w0: the first of the warp's 256 columns, whose draws its lanes make eight
// neighbours each; without VEC they then hand each other the results as bits.  drop: 1 by the draws, 2 none is kept.
template <bool VEC> struct Kept {
    uint4 w; uint32_t t;                             // VEC: the words, the threshold in the upper half; else the bits in w.x
    __device__ __forceinline__ void make(const DropoutParams &d, const PhiloxKeys &keys, int drop, int64_t base, int w0)
    {
        const int lane = threadIdx.x & 31;
        const uint64_t first = (uint64_t)(base + w0 + 8 * lane);
        t = d.threshold << 16;
        w = drop == 2 ? make_uint4(0u, 0u, 0u, 0u) : VEC ? dropout_block(d, keys, first >> 3) : dropout_draws8(d, keys, first);
        if (drop == 2) t = 0xFFFF0000u;
        if (VEC) return;
        uint32_t bits = 0, mine = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) bits |= (at_least(e) ? 1u : 0u) << e;
#pragma unroll
        for (int e = 0; e < 8; ++e) mine |= ((__shfl_sync(0xFFFFFFFFu, bits, 4 * e + (lane >> 3)) >> (lane & 7)) & 1u) << e;
        w.x = mine;
    }
    // (the high half of a word against the threshold: the word itself against it in the upper half)
    __device__ __forceinline__ bool at_least(int e) const
    {
        const uint32_t v = e < 2 ? w.x : e < 4 ? w.y : e < 6 ? w.z : w.w;
        return ((e & 1) ? v : v << 16) >= t;
    }
    __device__ __forceinline__ bool operator[](int e) const { return VEC ? at_least(e) : ((w.x >> e) & 1u) != 0; }
};

// Sums over the threads of a row's group, N at a time; every thread gets them.  WARP: the group is a warp.  `turn` alternates between
// the two halves of the scratch, so that one barrier an exchange is enough; `warps` take part.
constexpr int kJoinSums = 3;
typedef float JoinScratch[2][kJoinSums][16];
template <bool WARP, int N> __device__ __forceinline__ void group_sums(float (&v)[N], JoinScratch &scratch, int turn, int warps)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
        for (int n = 0; n < N; ++n) v[n] += __shfl_xor_sync(0xFFFFFFFFu, v[n], o);
    if (WARP) return;
    if ((threadIdx.x & 31) == 0) {
#pragma unroll
        for (int n = 0; n < N; ++n) scratch[turn][n][threadIdx.x >> 5] = v[n];
    }
    named_barrier(1, 32 * warps);
    // (every warp adds up the warps' sums by itself: one load a lane and four exchanges)
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = (int)(threadIdx.x & 15) < warps ? scratch[turn][n][threadIdx.x & 15] : 0.0f;
#pragma unroll
    for (int o = 8; o > 0; o >>= 1)
#pragma unroll
        for (int n = 0; n < N; ++n) v[n] += __shfl_xor_sync(0xFFFFFFFFu, v[n], o);
}
template <bool WARP> __device__ __forceinline__ float group_sum(float v, JoinScratch &scratch, int turn, int warps)
{
    float a[1] = {v};
    group_sums<WARP>(a, scratch, turn, warps);
    return a[0];
}

// The rows of an item: first, end.
struct ItemRows { int64_t gate, first, end; };
__device__ __forceinline__ ItemRows item_rows(const JoinItems &it, int64_t item)
{
    ItemRows r;
    r.gate = item / it.splits;
    r.first = r.gate * it.gate_rows + item % it.splits * it.split_rows;
    r.end = min(min(r.first + it.split_rows, (r.gate + 1) * it.gate_rows), it.rows);
    return r;
}

// A row's exchange of sums done, the next row's first one may write the half of the scratch that this row's last one is still read from,
// where a row has one sum only.
template <bool WARP> __device__ __forceinline__ void end_row(int pre, int post)
{
    if (!WARP && pre != post) __syncthreads();
}

// ---- rows read in vectors, through the ring ------------------------------------------------------------------------------
// A row is copied by a lane of its group's first warp, whose bytes a slot's barrier reports (full).  Forward a slot is free for the next
// copy once its row's sums have been exchanged; backwards, where a row is read behind the exchange too, each warp says so (empty).  Every wait
// is bounded: a warp whose wait ran out raises the status word, gives copies in flight another millisecond, copies and waits for nothing any
// more and goes through the rest of its rows for the block's barriers' sake.
template <typename T> struct Pieces { static constexpr int n = sizeof(T) / 2; };
constexpr int kJoinSlots = 3, kJoinBackSlots = 2;
struct JoinBars { uint64_t full[kJoinWarpRows][kJoinSlots], empty[kJoinBackSlots]; };
__device__ __forceinline__ void join_bars_init(JoinBars &bars, int warps)
{
    if (threadIdx.x == 0) {
        for (int w = 0; w < kJoinWarpRows; ++w)
            for (int k = 0; k < kJoinSlots; ++k) mbar_init(&bars.full[w][k], 1);
        for (int k = 0; k < kJoinBackSlots; ++k) mbar_init(&bars.empty[k], (uint32_t)warps);
        mbar_fence_init();
    }
    __syncthreads();
}
struct JoinSource { const void *row0; uint32_t row_bytes, offset; };        // offset: of the tensor's row in a slot
// One row of each tensor into a slot, by a converged warp.
template <int N> __device__ __forceinline__ void join_copy(uint8_t *slot, uint64_t *full, const JoinSource (&src)[N], int64_t row)
{
    if (elect_one()) {
        uint32_t bytes = 0;
#pragma unroll
        for (int k = 0; k < N; ++k) bytes += src[k].row0 ? src[k].row_bytes : 0u;
        mbar_expect_tx(full, bytes);
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (src[k].row0) bulk_load(slot + src[k].offset, static_cast<const char *>(src[k].row0) + row * src[k].row_bytes, src[k].row_bytes, full);
    }
    __syncwarp();
}
// A warp's place in a ring of slots.
struct JoinPlace {
    uint32_t slot, ph;
    __device__ __forceinline__ JoinPlace next(uint32_t slots) const { return slot + 1 == slots ? JoinPlace{0u, ph ^ 1u} : JoinPlace{slot + 1, ph}; }
};
__device__ __forceinline__ void join_wait(uint64_t *bar, uint32_t parity, bool &dead, int *status)
{
    if (!dead && !mbar_wait_uniform(bar, parity)) { dead = true; raise_timeout(status); __nanosleep(1000000); }
}
// Eight columns of a row in a slot (zero behind the last one).
template <typename T> __device__ __forceinline__ void ring_read(const uint8_t *row, int c, bool in, float (&v)[8])
{
    Raw8<T> r;
    const uint4 *p = reinterpret_cast<const uint4 *>(row + c * (int)sizeof(T));
#pragma unroll
    for (int i = 0; i < Pieces<T>::n; ++i) r.w[i] = in ? p[i] : make_uint4(0, 0, 0, 0);
    unpack8(r, v);
}
// (wide: fp32 rows start on 32-byte boundaries)
template <typename T> __device__ __forceinline__ void put_vec(void *row0, int64_t at, const Raw8<T> &r, int wide)
{
    uint4 *p = reinterpret_cast<uint4 *>(static_cast<T *>(row0) + at);
    if (Pieces<T>::n == 2 && wide) put32(p, r.w[0], r.w[Pieces<T>::n - 1]);
    else {
#pragma unroll
        for (int i = 0; i < Pieces<T>::n; ++i) p[i] = r.w[i];
    }
}
// gate * w_post of eight columns (zero behind the last one)
__device__ __forceinline__ void join_gains(const float *gate, const float *w_post, int64_t gate_at, int c, bool in, float (&v)[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 1.0f;
    if (!in) return;
    if (gate) unpack8(load8(gate + gate_at + c, 8, true), v);
    if (w_post) {
        float w[8];
        unpack8(load8(w_post + c, 8, true), w);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= w[e];
    }
}

template <typename TX, typename TB, int CH, bool WARP, int MAXT>
__global__ void __launch_bounds__(MAXT, MAXT == 256 ? 2 : 1)
join_fwd_kernel(const __grid_constant__ JoinParams P, const __grid_constant__ PhiloxKeys keys)
{
    extern __shared__ __align__(16) uint8_t ring[];
    __shared__ JoinScratch scratch;
    __shared__ JoinBars bars;
    const int lane = threadIdx.x & 31, all_warps = (int)(blockDim.x >> 5), warp = WARP ? 0 : threadIdx.x >> 5, warps = WARP ? 1 : all_warps;
    const int sub = WARP ? threadIdx.x >> 5 : 0, subs = WARP ? kJoinWarpRows : 1;
    const int cols = (int)P.it.cols, c0 = 256 * warp + 8 * lane, apart = 256 * warps;      // the thread's first column, and its next ones'
    const uint32_t row_x = (uint32_t)cols * sizeof(TX), row_b = (uint32_t)cols * sizeof(TB), slot_bytes = row_x + row_b;
    join_bars_init(bars, all_warps);
    pdl_wait();
    if (blockIdx.x == 0 && threadIdx.x == 0) *P.status = 0;          // (a wait gives up a second later at the earliest)
    uint8_t *const slots = ring + (uint32_t)(sub * kJoinSlots) * slot_bytes;
    uint64_t *const full = bars.full[sub];
    const JoinSource src[2] = {{P.x, row_x, 0u}, {P.b, row_b, row_x}};
    bool dead = false;
    const auto fetch = [&](int64_t row, int64_t end, uint32_t slot) {
        if ((WARP || warp == 0) && row < end && !dead) join_copy<2>(slots + slot * slot_bytes, &full[slot], src, row);
    };
    bool in[CH];
    float gw[CH][8], w2[CH][8];
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        in[k] = c0 + k * apart < cols;
        join_gains(P.w_pre, nullptr, 0, c0 + k * apart, in[k], w2[k]);
    }
    const auto square_sum = [&](uint32_t slot) {
        float s = 0.0f;
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            float v[8];
            ring_read<TB>(slots + slot * slot_bytes + row_x, c0 + k * apart, in[k], v);
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
            for (int k = 0; k < CH; ++k) join_gains(P.gate, P.post ? P.w_post : nullptr, rows.gate * cols, c0 + k * apart, in[k], gw[k]);
            had = rows.gate;
        }
        // (all slots are free: the last rows' sums have been exchanged)
        JoinPlace p = place;
        for (int k = 0; k < kJoinSlots; ++k) { fetch(rows.first + sub + k * subs, rows.end, p.slot); p = p.next(kJoinSlots); }
        float rstd = 1.0f;
        if (rows.first + sub < rows.end) {
            join_wait(&full[place.slot], place.ph, dead, P.status);
            if (P.post) { rstd = rsqrtf(group_sum<WARP>(square_sum(place.slot), scratch, half, warps) * P.inv_cols + P.eps); half ^= 1; }
        }
        for (int64_t row = rows.first + sub; row < rows.end; row += subs) {
            const int64_t at = row * cols + c0;
            const float scale = factor * rstd;
            float r[CH][8], sums[2] = {0.0f, 0.0f};           // of this row's r^2, of the next row's b^2
            if (P.post && P.rstd_post && warp == 0 && lane == 0) P.rstd_post[row] = rstd;
            {
#pragma unroll
                for (int k = 0; k < CH; ++k) {
                    ring_read<TX>(slots + place.slot * slot_bytes, c0 + k * apart, in[k], r[k]);
#pragma unroll
                    for (int e = 0; e < 8; ++e) r[k][e] *= P.alpha;
                    if (P.b) {
                        float b[8];
                        ring_read<TB>(slots + place.slot * slot_bytes + row_x, c0 + k * apart, in[k], b);
                        if (P.drop) {                 // (what is dropped counts for nothing, whatever it is: chosen, not multiplied by zero)
                            Kept<true> kept;
                            kept.make(P.d, keys, P.drop, at - 8 * lane + k * apart, 0);
#pragma unroll
                            for (int e = 0; e < 8; ++e) b[e] = kept[e] ? b[e] : 0.0f;
                        }
#pragma unroll
                        for (int e = 0; e < 8; ++e) r[k][e] = fmaf(b[e] * scale, gw[k][e], r[k][e]);
                    }
                    const Raw8<TX> raw = pack8<TX>(r[k]);
                    if (P.r && in[k]) put_vec(P.r, at + k * apart, raw, P.wide);
                    unpack8(raw, r[k]);
#pragma unroll
                    for (int e = 0; e < 8; ++e) sums[0] = fmaf(r[k][e], r[k][e], sums[0]);    // (zero behind the last column, as x and b are)
                }
            }
            const JoinPlace following = place.next(kJoinSlots);
            if (row + subs < rows.end) {
                join_wait(&full[following.slot], following.ph, dead, P.status);
                if (P.post) sums[1] = square_sum(following.slot);
            }
            __syncwarp();
            group_sums<WARP>(sums, scratch, half, warps);
            half ^= 1;
            fetch(row + kJoinSlots * subs, rows.end, place.slot);
            place = following;
            rstd = P.post ? rsqrtf(sums[1] * P.inv_cols + P.eps) : 1.0f;
            if (P.pre) {
                const float rstd2 = rsqrtf(sums[0] * P.inv_cols + P.eps);
                if (P.rstd_pre && warp == 0 && lane == 0) P.rstd_pre[row] = rstd2;
#pragma unroll
                for (int k = 0; k < CH; ++k) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) r[k][e] = r[k][e] * rstd2 * w2[k][e];
                    if (in[k]) put_vec(P.h, at + k * apart, pack8<TB>(r[k]), P.wide);
                }
            }
        }
    }
}

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

template <typename TX, typename TB, int CH, bool WARP, int MAXT>
__global__ void __launch_bounds__(MAXT, MAXT == 256 && !WARP ? 2 : 1)
join_bwd_kernel(const __grid_constant__ JoinBwdParams P, const __grid_constant__ PhiloxKeys keys)
{
    extern __shared__ __align__(16) uint8_t ring[];
    __shared__ float fold[WARP ? kJoinWarpRows * 256 * CH : 1];            // WARP: the warps' sums
    __shared__ JoinScratch scratch;
    __shared__ JoinBars bars;
    const int lane = threadIdx.x & 31, all_warps = (int)(blockDim.x >> 5), warp = WARP ? 0 : threadIdx.x >> 5, warps = WARP ? 1 : all_warps;
    const int sub = WARP ? threadIdx.x >> 5 : 0, subs = WARP ? kJoinWarpRows : 1;
    const int cols = (int)P.it.cols, c0 = 256 * warp + 8 * lane, apart = 256 * warps;
    const uint32_t row_x = (uint32_t)cols * sizeof(TX), row_b = (uint32_t)cols * sizeof(TB);
    const uint32_t off_h = 2u * row_x, off_b = off_h + row_b, slot_bytes = off_b + row_b;          // dr, r, dh, b
    join_bars_init(bars, all_warps);
    pdl_wait();
    if (blockIdx.x == 0 && threadIdx.x == 0) *P.status = 0;          // (a wait gives up a second later at the earliest)
    uint8_t *const slots = ring + (uint32_t)(sub * kJoinBackSlots) * slot_bytes;
    uint64_t *const full = bars.full[sub];
    const JoinSource src[4] = {{P.dr, row_x, 0u}, {P.pre ? P.r : nullptr, row_x, row_x}, {P.pre ? P.dh : nullptr, row_b, off_h}, {P.b, row_b, off_b}};
    bool dead = false;
    JoinPlace place{0u, 0u}, ahead{0u, 1u};          // of the row at hand, of the next row to be copied
    const auto fetch = [&](int64_t row) {
        if (WARP || warp == 0) {
            if (!WARP) join_wait(&bars.empty[ahead.slot], ahead.ph, dead, P.status);
            if (!dead) join_copy<4>(slots + ahead.slot * slot_bytes, &full[ahead.slot], src, row);
            ahead = ahead.next(kJoinBackSlots);
        }
    };
    bool in[CH];
    float gw[CH][8], w2[CH][8], a_pre[CH][8] = {};
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        in[k] = c0 + k * apart < cols;
        join_gains(P.w_pre, nullptr, 0, c0 + k * apart, in[k], w2[k]);
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
        for (int k = 0; k < CH; ++k) join_gains(P.gate, P.post ? P.w_post : nullptr, rows.gate * cols, c0 + k * apart, in[k], gw[k]);
        if (rows.first + sub < rows.end) fetch(rows.first + sub);
        for (int64_t row = rows.first + sub; row < rows.end; row += subs) {
            const int64_t at = row * cols + c0;
            const float rstd1 = next1, rstd2 = next2;
            if (row + subs < rows.end) {
                if (P.post) next1 = __ldg(P.rstd_post + row + subs);
                if (P.pre) next2 = __ldg(P.rstd_pre + row + subs);
                fetch(row + subs);
            }
            join_wait(&full[place.slot], place.ph, dead, P.status);
            const uint8_t *const my_g = slots + place.slot * slot_bytes, *const my_r = my_g + row_x, *const my_h = my_g + off_h, *const my_b = my_g + off_b;
            const auto get_g = [&](int k, float (&v)[8]) { ring_read<TX>(my_g, c0 + k * apart, in[k] && P.dr, v); };
            const auto get_r = [&](int k, float (&v)[8]) { ring_read<TX>(my_r, c0 + k * apart, in[k] && P.pre, v); };
            const auto get_h = [&](int k, float (&v)[8]) { ring_read<TB>(my_h, c0 + k * apart, in[k] && P.pre, v); };
            const auto get_b = [&](int k, float (&v)[8]) { ring_read<TB>(my_b, c0 + k * apart, in[k] && P.b, v); };
            // Both means from one exchange: the second, of v w_post b, is linear in the first, m, with R = (dr + dh w_pre rstd_pre) - r m.
            float sums[3] = {0.0f, 0.0f, 0.0f};
            uint32_t kept = 0;                        // which elements the dropout keeps, a bit each
            {
#pragma unroll
                for (int k = 0; k < CH; ++k) {
                    float h[8], r[8], g[8], b[8];
                    get_h(k, h); get_r(k, r); get_g(k, g); get_b(k, b);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        a_pre[k][e] = fmaf(h[e] * r[e], rstd2, a_pre[k][e]);
                        h[e] *= w2[k][e];
                        sums[0] = fmaf(h[e], r[e], sums[0]);
                        b[e] *= gw[k][e];
                    }
                    if (P.drop) {
                        Kept<true> q;
                        q.make(P.d, keys, P.drop, at - 8 * lane + k * apart, 0);
#pragma unroll
                        for (int e = 0; e < 8; ++e) { const bool on = q[e]; kept |= on ? 1u << (8 * k + e) : 0u; b[e] = on ? b[e] : 0.0f; }
                    }
                    if (P.post) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            sums[1] = fmaf(fmaf(h[e], rstd2, g[e]), b[e], sums[1]);
                            sums[2] = fmaf(r[e], b[e], sums[2]);
                        }
                    }
                }
            }
            if (P.pre || P.post) { group_sums<WARP>(sums, scratch, half, warps); half ^= 1; }
            // R = dr + rstd2 (dh w_pre) - r m2;  db = z rstd1 - b m1 with z = R dropout' gate w_post
            const float m2 = P.pre ? sums[0] * P.inv_cols * rstd2 * rstd2 * rstd2 : 0.0f;
            const float m1 = P.post ? (sums[1] - m2 * sums[2]) * factor * P.inv_cols * rstd1 * rstd1 * rstd1 : 0.0f;
            const float f1 = factor * rstd1;
            {
#pragma unroll
                for (int k = 0; k < CH; ++k) {
                    float R[8];
                    get_g(k, R);
                    if (P.pre) {
                        float h[8], r[8];
                        get_h(k, h); get_r(k, r);
#pragma unroll
                        for (int e = 0; e < 8; ++e) R[e] = fmaf(-r[e], m2, fmaf(h[e] * w2[k][e], rstd2, R[e]));
                    }
                    if (P.b) {
                        float b[8], z[8];
                        get_b(k, b);
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
                        if (P.db && in[k]) {
#pragma unroll
                            for (int e = 0; e < 8; ++e) z[e] = P.post ? fmaf(-b[e], m1, z[e] * gw[k][e]) : z[e] * gw[k][e];
                            put_vec(P.db, at + k * apart, pack8<TB>(z), P.wide);
                        }
                    }
                    if (P.dx && in[k]) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) R[e] *= P.alpha;
                        put_vec(P.dx, at + k * apart, pack8<TX>(R), P.wide);
                    }
                }
            }
            __syncwarp();
            if (!WARP && lane == 0) mbar_arrive(&bars.empty[place.slot]);
            place = place.next(kJoinBackSlots);
        }
        if (P.sum_gate) join_leave<CH, WARP, true>(S, P.part_gate + item * cols, P.post ? P.w_post : nullptr, cols, c0, apart, false, fold, 32 * all_warps);
        if (P.sum_post)
            join_leave<CH, WARP, true>(S, P.part_post + (int64_t)blockIdx.x * cols, P.gate ? P.gate + rows.gate * cols : nullptr, cols, c0, apart, item != blockIdx.x, fold, 32 * all_warps);
    }
    if (P.sum_pre) join_leave<CH, WARP, true>(a_pre, P.part_pre + (int64_t)blockIdx.x * cols, nullptr, cols, c0, apart, false, fold, 32 * all_warps);
}

// ---- any rows -------------------------------------------------------------------------------------------------------------
template <typename TX, typename TB, int CH> struct JoinRow { Held<TX> x[CH]; Held<TB> b[CH]; };

template <typename TX, typename TB, int CH, bool WARP, bool VEC>
__global__ void __launch_bounds__(WARP ? 32 * kJoinWarpRows : 512, 1)
join_fwd_any_kernel(const __grid_constant__ JoinParams P, const __grid_constant__ PhiloxKeys keys)
{
    __shared__ JoinScratch scratch;
    const int lane = threadIdx.x & 31, warp = WARP ? 0 : threadIdx.x >> 5, warps = WARP ? 1 : blockDim.x >> 5;
    const int sub = WARP ? threadIdx.x >> 5 : 0, subs = WARP ? kJoinWarpRows : 1;
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
        for (int64_t row = rows.first + sub; row < rows.end; row += subs) {
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
                rstd = rsqrtf(group_sum<WARP>(s, scratch, 0, warps) * P.inv_cols + P.eps);
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
                const float rstd2 = rsqrtf(group_sum<WARP>(s2, scratch, 1, warps) * P.inv_cols + P.eps);
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
            end_row<WARP>(P.pre, P.post);
        }
    }
}

template <typename TX, typename TB, int CH> struct JoinBwdRow { Held<TX> g[CH], r[CH]; Held<TB> h[CH], b[CH]; };

template <typename TX, typename TB, int CH, bool WARP, bool VEC>
__global__ void __launch_bounds__(WARP ? 32 * kJoinWarpRows : 512, 1)
join_bwd_any_kernel(const __grid_constant__ JoinBwdParams P, const __grid_constant__ PhiloxKeys keys)
{
    __shared__ float fold[WARP ? kJoinWarpRows * 256 * CH : 1];
    __shared__ JoinScratch scratch;
    const int lane = threadIdx.x & 31, warp = WARP ? 0 : threadIdx.x >> 5, warps = WARP ? 1 : blockDim.x >> 5;
    const int sub = WARP ? threadIdx.x >> 5 : 0, subs = WARP ? kJoinWarpRows : 1;
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
        for (int64_t row = rows.first + sub; row < rows.end; row += subs) {
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
                mean2 = group_sum<WARP>(s, scratch, 0, warps) * P.inv_cols;
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
                const float mean1 = P.post ? group_sum<WARP>(s1, scratch, 1, warps) * P.inv_cols * rstd1 : 0.0f;
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
            end_row<WARP>(P.pre, P.post);
        }
        if (P.sum_gate) join_leave<CH, WARP, VEC>(S, P.part_gate + item * (int64_t)cols, P.post ? P.w_post : nullptr, cols, col(0), 256 * warps, false, fold, (int)blockDim.x);
        if (P.sum_post)
            join_leave<CH, WARP, VEC>(S, P.part_post + (int64_t)blockIdx.x * cols, P.gate ? P.gate + rows.gate * (int64_t)cols : nullptr, cols, col(0), 256 * warps,
                                      item != blockIdx.x, fold, (int)blockDim.x);
    }
    if (P.sum_pre) join_leave<CH, WARP, VEC>(a_pre, P.part_pre + (int64_t)blockIdx.x * cols, nullptr, cols, col(0), 256 * warps, false, fold, (int)blockDim.x);
}
#endif

// out[o][c] = sum over `count` partial rows in [outs][count][cols], in a fixed order: the thirty-two warps of a block take every
// thirty-second row, 32 V columns of it, eight loads at a time (a sum waits for its loads and for nothing else), then the thirty-two are
// added up.  V: 4 where rows are whole groups of four floats (293 rows of 4096, three times: 11.1 us; one column a lane 14.7 us).
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
struct JoinShape { int ch, threads; bool warp; };
constexpr size_t kJoinMaxRing = 200 * 1024, kJoinSmRings = 222 * 1024;        // of a block, of an SM
// Shared memory of a block's ring: forward slots of one tensor of each type, backwards of two.
static size_t join_ring(const qbp_resnorm_desc *d, const JoinShape &s, int tensors)
{
    const size_t slots = tensors == 1 ? kJoinSlots : kJoinBackSlots;
    return slots * (size_t)(s.warp ? kJoinWarpRows : 1) * (size_t)d->cols * (size_t)tensors * (dtype_size(d->x_dtype) + dtype_size(d->b_dtype));
}
// A thread takes sixteen columns, eight where the rings of two blocks would not fit an SM, and 32 (without a ring) beyond 8192.
static JoinShape join_shape(const qbp_resnorm_desc *d, int tensors)
{
    const int chunks = (int)((d->cols + 255) / 256);                 // a warp's eight columns a lane
    if (chunks <= 1) return {1, 32 * kJoinWarpRows, true};
    if (chunks <= 2) return {2, 32 * kJoinWarpRows, true};
    JoinShape s{2, 32 * ((chunks + 1) / 2), false};
    if (s.threads > 128 && chunks <= 16 && 2 * join_ring(d, s, tensors) > kJoinSmRings) s = {1, 32 * chunks, false};
    if (s.threads <= 512 && join_ring(d, s, tensors) <= kJoinMaxRing) return s;
    return {4, 32 * ((chunks + 3) / 4), false};
}

// Runs `call` with the kernel's compile-time choices for rows that are read in vectors.
#define QBP_FOR_JOIN(shape, CH, WARP, MAXT, call)                                                                             \
    do {                                                                                                                      \
        if ((shape).warp && (shape).ch == 1) { constexpr int CH = 1, MAXT = 256; constexpr bool WARP = true; call; }          \
        else if ((shape).warp) { constexpr int CH = 2, MAXT = 256; constexpr bool WARP = true; call; }                        \
        else if ((shape).ch == 1) { constexpr int CH = 1, MAXT = 512; constexpr bool WARP = false; call; }                    \
        else if ((shape).threads <= 256) { constexpr int CH = 2, MAXT = 256; constexpr bool WARP = false; call; }             \
        else { constexpr int CH = 2, MAXT = 512; constexpr bool WARP = false; call; }                                         \
    } while (0)

// Launches with the ring's shared memory.
template <typename Params>
static int launch_join(void (*kernel)(Params, PhiloxKeys), PerDeviceOnce &once, int64_t blocks, const JoinShape &s, size_t smem, cudaStream_t st, const Params &P,
                       const PhiloxKeys &keys)
{
    if (smem > 24 * 1024) QBP_SMEM_OPT_IN(once, kernel, kJoinMaxRing);       // (with the static arrays beside it, over 48 KB)
    launch(kernel, dim3((unsigned)blocks), s.threads, smem, st, P, keys);
    return QBP_OK;
}

static int check_join(const qbp_resnorm_desc *d, const char *name, const void *b, const float *gate, const float *w_post, const float *w_pre)
{
    if (!d) return fail(QBP_ERR_INVALID_ARG, "%s: NULL descriptor", name);
    if (!dtype_ok(d->x_dtype) || !dtype_ok(d->b_dtype)) return fail(QBP_ERR_INVALID_ARG, "%s: dtypes %d and %d", name, d->x_dtype, d->b_dtype);
    if (d->rows < 0 || d->cols < 0 || d->gate_rows < 0) return fail(QBP_ERR_INVALID_ARG, "%s: rows %lld, cols %lld, gate_rows %lld", name, (long long)d->rows, (long long)d->cols, (long long)d->gate_rows);
    if (d->cols > kJoinMaxCols) return fail(QBP_ERR_UNSUPPORTED_SHAPE, "%s: %lld columns, at most %lld", name, (long long)d->cols, (long long)kJoinMaxCols);
    if (!(d->eps >= 0.0f) || !(d->p >= 0.0f && d->p <= 1.0f) || std::isinf(d->eps)) return fail(QBP_ERR_INVALID_ARG, "%s: eps %g, p %g", name, (double)d->eps, (double)d->p);
    if (d->index_base % 8) return fail(QBP_ERR_INVALID_ARG, "%s: index_base %llu is not a multiple of 8", name, (unsigned long long)d->index_base);
    if (!b && d->rows > 0 && d->cols > 0 && (d->post || gate || d->p > 0.0f)) return fail(QBP_ERR_INVALID_ARG, "%s: a norm after, a gate or dropout without a block output", name);
    for (const float *w : {gate, w_post, w_pre})
        if (!aligned_to(w, 4)) return fail(QBP_ERR_INVALID_ARG, "%s: misaligned parameters", name);
    return QBP_OK;
}
// A call with nothing to do (a workspace that is there gets its status word cleared all the same).
static int join_empty(void *ws, size_t ws_bytes, cudaStream_t st)
{
    if (ws && aligned_to(ws, 4) && ws_bytes >= 4) QBP_CUDA_OK(cudaMemsetAsync(ws, 0, 4, st));
    return QBP_OK;
}
static bool real_ok(const void *p, int dtype) { return p && aligned_to(p, dtype_size(dtype)); }
static int64_t join_gates(const qbp_resnorm_desc *d) { return d->gate_rows ? (d->rows + d->gate_rows - 1) / d->gate_rows : 1; }

// How the rows are cut for a grid of at most `most` blocks: items of neighbouring rows of one gate.
struct JoinCut { JoinItems it; int64_t blocks; };
static JoinCut join_cut(const qbp_resnorm_desc *d, const JoinShape &s, bool per_gate, int64_t most, int64_t few)
{
    JoinCut c{};
    JoinItems &it = c.it;
    it.rows = d->rows; it.cols = d->cols;
    it.gates = per_gate && d->gate_rows ? join_gates(d) : 1;
    it.gate_rows = per_gate && d->gate_rows ? d->gate_rows : std::max<int64_t>(d->rows, 1);
    if (s.warp) few *= kJoinWarpRows;                                // a block takes so many rows at a time
    it.splits = std::max<int64_t>(1, std::min((most + it.gates - 1) / it.gates, (it.gate_rows + few - 1) / few));
    it.split_rows = (it.gate_rows + it.splits - 1) / it.splits;
    it.splits = (it.gate_rows + it.split_rows - 1) / it.split_rows;
    c.blocks = std::min(most, it.gates * it.splits);
    return c;
}
// Partial rows of dgate: none where an item is all of a gate's rows, whose sum is the gradient.
static size_t gate_parts(const JoinItems &it) { return it.splits > 1 ? (size_t)(it.gates * it.splits * it.cols) : 0; }
// Blocks of a wave: 16 warps an SM (8 backwards where a row is a warp's), which their registers allow, or what their rings leave room for.
static int64_t join_blocks(const qbp_resnorm_desc *d, const JoinShape &s, int tensors)
{
    const int64_t per_sm = s.ch > 2 ? 1 : std::min<int64_t>((s.warp && tensors == 2 ? 256 : 512) / s.threads, (int64_t)(227 * 1024 / (join_ring(d, s, tensors) + 2048 + (s.warp && tensors == 2 ? 16384 : 0))));
    return (int64_t)sm_count() * std::max<int64_t>(per_sm, 1);
}
static JoinCut join_cut_bwd(const qbp_resnorm_desc *d, bool per_gate)
{
    const JoinShape s = join_shape(d, 2);
    return join_cut(d, s, per_gate, join_blocks(d, s, 2), s.warp ? 2 : 4);
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
    const JoinShape s = join_shape(d, 1);
    const JoinCut c = join_cut(d, s, gate != nullptr, join_blocks(d, s, 1), 1);
    P.it = c.it;
    P.x = x; P.b = b; P.w_post = w_post; P.gate = gate; P.w_pre = w_pre; P.r = r; P.h = h; P.rstd_post = rstd_post; P.rstd_pre = rstd_pre;
    P.eps = d->eps; P.alpha = d->alpha; P.inv_cols = (float)(1.0 / (double)d->cols);
    P.post = d->post ? 1 : 0; P.pre = d->pre ? 1 : 0; P.x_dtype = d->x_dtype; P.b_dtype = d->b_dtype;
    P.d = dropout_params(d->p, d->tensor_id, d->index_base);
    P.drop = P.d.threshold == 65536u ? 2 : P.d.threshold ? 1 : 0;
    P.status = static_cast<int *>(ws);
    P.wide = aligned_to(r, 32) && aligned_to(h, 32) ? 1 : 0;
    const PhiloxKeys keys = philox_keys_host(d->seed);
    const bool vec = d->cols % 8 == 0 && aligned16(x) && aligned16(b) && aligned16(r) && aligned16(h) && aligned16(w_post) && aligned16(gate) && aligned16(w_pre);
    QBP_TRACE_BEGIN(st);
    if (vec && s.ch <= 2)
        QBP_FOR_DTYPE(d->x_dtype, TX, QBP_FOR_DTYPE(d->b_dtype, TB, QBP_FOR_JOIN(s, CH, WARP, MAXT, {
            static PerDeviceOnce once;
            if ((rc = launch_join(join_fwd_kernel<TX, TB, CH, WARP, MAXT>, once, c.blocks, s, join_ring(d, s, 1), st, P, keys))) return rc;
        })));
    else if (vec)
        QBP_FOR_DTYPE(d->x_dtype, TX, QBP_FOR_DTYPE(d->b_dtype, TB, (launch(join_fwd_any_kernel<TX, TB, 4, false, true>, dim3((unsigned)c.blocks), s.threads, 0, st, P, keys))));
    else if (s.ch == 4)
        launch(join_fwd_any_kernel<AnyReal, AnyReal, 4, false, false>, dim3((unsigned)c.blocks), s.threads, 0, st, P, keys);
    else
        QBP_FOR_JOIN(s, CH, WARP, MAXT, (launch(join_fwd_any_kernel<AnyReal, AnyReal, CH, WARP, false>, dim3((unsigned)c.blocks), s.threads, 0, st, P, keys)));
    QBP_LAUNCH_OK("join_fwd_kernel");
    return QBP_OK;
}

extern "C" __attribute__((visibility("default"))) size_t qbp_resnorm_bwd_workspace_bytes(const qbp_resnorm_desc *d)
{
    if (!d || d->rows <= 0 || d->cols <= 0) return 256;
    size_t most = 0;
    for (bool per_gate : {false, true}) {
        const JoinCut c = join_cut_bwd(d, per_gate);
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
    const JoinCut c = join_cut_bwd(d, gate || dgate);
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
    P.wide = aligned_to(dx, 32) && aligned_to(db, 32) ? 1 : 0;
    const PhiloxKeys keys = philox_keys_host(d->seed);
    const JoinShape s = join_shape(d, 2);
    const bool vec = d->cols % 8 == 0 && aligned16(dr) && aligned16(dh) && aligned16(b) && aligned16(r) && aligned16(dx) && aligned16(db) && aligned16(w_post) &&
                     aligned16(gate) && aligned16(w_pre);
    QBP_TRACE_BEGIN(st);
    if (vec && s.ch <= 2)
        QBP_FOR_DTYPE(d->x_dtype, TX, QBP_FOR_DTYPE(d->b_dtype, TB, QBP_FOR_JOIN(s, CH, WARP, MAXT, {
            static PerDeviceOnce once;
            if ((rc = launch_join(join_bwd_kernel<TX, TB, CH, WARP, MAXT>, once, c.blocks, s, join_ring(d, s, 2), st, P, keys))) return rc;
        })));
    else if (vec)
        QBP_FOR_DTYPE(d->x_dtype, TX, QBP_FOR_DTYPE(d->b_dtype, TB, (launch(join_bwd_any_kernel<TX, TB, 4, false, true>, dim3((unsigned)c.blocks), s.threads, 0, st, P, keys))));
    else if (s.ch == 4)
        launch(join_bwd_any_kernel<AnyReal, AnyReal, 4, false, false>, dim3((unsigned)c.blocks), s.threads, 0, st, P, keys);
    else
        QBP_FOR_JOIN(s, CH, WARP, MAXT, (launch(join_bwd_any_kernel<AnyReal, AnyReal, CH, WARP, false>, dim3((unsigned)c.blocks), s.threads, 0, st, P, keys)));
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
