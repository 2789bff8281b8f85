// The join between two blocks of a residual network and its gradients (include/qbp.h; qbp_resnorm_fwd in qbp_resnorm.cu, qbp_resnorm_bwd in
// qbp_resnorm_bwd.cu): what both use.  Norm after a block, gate, dropout, residual stream and the norm before the next block, in one pass over
// the rows.
//
// A row is held in registers by the threads of one group: a warp (of a block's eight) for rows of up to 512 columns, a block of up to 512
// threads beyond; a thread has CH times eight columns.  The two sums over a row (of b^2 and of r^2; backwards of the gradients' projections on
// r and b) are exchanged between the group's threads, forward a row's second with the next row's first, backwards both at once, and nothing
// is read from memory twice.  A block takes neighbouring rows of one gate (an item) and keeps the parameters of its columns in registers.  Rows
// come through a ring of two or three in shared memory, copied whole by one thread (cp.async.bulk): a row is on its way while the one before is
// worked on, and stays out of the threads' registers.  (Copied by the threads that read it, 16 bytes each, a row of 48 KB took 2100 cycles of
// their time, of 5900.)  16384 x 4096, fp32 stream, bf16 blocks, dropout: forward 142 us, 5.7 TB/s, backward 197 us, 6.1 TB/s.
//
// Backwards, with gate and w_post constant along an item's columns, dw_post and dgate are multiples of one sum over its rows,
// S = sum of R dropout'(b rstd_post): dgate = w_post S, dw_post = gate S.  A thread keeps S and dw_pre's sum in registers, a block leaves
// one partial row of each, and a second kernel adds these up in a fixed order.
//
// Columns.  Rows that all start on 16-byte boundaries are read from the ring eight neighbouring columns to a thread (VEC).  Others are copied
// from the 16-byte boundary before them and read element by element, the lanes of a warp side by side.  Beyond 8192 columns, or where the rings
// find no room, the rows are read from memory by the threads that use them (the _wide kernels).
#pragma once

#include "qbp_dropout.cuh"

#include <algorithm>
#include <limits>

namespace qbp {

constexpr int kJoinWarpRows = 8;                    // rows of a block whose groups are warps
constexpr int64_t kJoinMaxCols = QBP_RESNORM_MAX_COLS;

// How the rows are cut: `gates` gates of `gate_rows` rows, each in `splits` items of `split_rows` rows (the last one fewer).
struct JoinItems { int64_t rows, cols, gate_rows, gates, splits, split_rows; };

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

// ---- rows through the ring -----------------------------------------------------------------------------------------------
// A row is copied by a lane of its group's first warp, whose bytes a slot's barrier reports (full).  A slot is free for the next copy once
// its row's sums have been exchanged; backwards with sixteen columns a thread, where a row is read behind the exchange too, each warp says so (empty).  Every wait
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
__device__ __forceinline__ void mbar_expect_bytes(uint64_t *bar, uint32_t bytes)
{
    asm volatile("mbarrier.expect_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}
struct JoinSource { const void *row0; uint32_t row_bytes, offset; };        // offset: of the tensor's row in a slot
// Bytes of a slot for a tensor's row: the row, or without VEC from the 16-byte boundary before it to the one behind it.
template <bool VEC> __host__ __device__ constexpr uint32_t join_section(uint32_t row_bytes) { return VEC ? row_bytes : ((row_bytes + 15u) & ~15u) + 16u; }
// How far behind its section's start a row begins.
__device__ __forceinline__ uint32_t join_shift(const JoinSource &s, int64_t row) { return ((uint32_t)reinterpret_cast<uintptr_t>(s.row0) + (uint32_t)row * s.row_bytes) & 15u; }
// A row off the 16-byte boundaries, by one lane: the 16-byte pieces that lie within the tensor as one copy, the others, which hold the
// tensor's first or last elements, by hand (and fenced: the slot's next row is copied over them by the asynchronous proxy, ahead of which
// barriers alone order no ordinary store).
template <typename T> __device__ __forceinline__ void join_copy_from_before(uint8_t *section, uint64_t *full, const JoinSource &s, int64_t row, int64_t rows)
{
    const uintptr_t first = reinterpret_cast<uintptr_t>(s.row0), a = first + (uintptr_t)(row * s.row_bytes), e = a + s.row_bytes, base = a & ~(uintptr_t)15;
    uintptr_t lo = base, hi = (e + 15) & ~(uintptr_t)15;
    if (row == 0 || row == rows - 1 || s.row_bytes < 32) {           // (no other row reaches over the tensor's ends)
        lo = max(lo, (first + 15) & ~(uintptr_t)15); hi = min(hi, (first + (uintptr_t)(rows * s.row_bytes)) & ~(uintptr_t)15);
        for (uintptr_t p = a; p < min(e, lo); p += sizeof(T)) *reinterpret_cast<T *>(section + (p - base)) = *reinterpret_cast<const T *>(p);
        for (uintptr_t p = max(a, hi); p < e; p += sizeof(T)) *reinterpret_cast<T *>(section + (p - base)) = *reinterpret_cast<const T *>(p);
        fence_proxy_async();
        if (lo >= hi) return;
    }
    mbar_expect_bytes(full, (uint32_t)(hi - lo));
    bulk_load(section + (lo - base), reinterpret_cast<const void *>(lo), (uint32_t)(hi - lo), full);
}
// One row of each tensor into a slot, by a converged warp.  The first TXS tensors are of type TX, the others of type TB.
template <typename TX, typename TB, int TXS, bool VEC, int N>
__device__ __forceinline__ void join_copy(uint8_t *slot, uint64_t *full, const JoinSource (&src)[N], int64_t row, int64_t rows)
{
    if (elect_one()) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            if (!src[k].row0) continue;
            uint8_t *const section = slot + src[k].offset;
            if (VEC) {
                mbar_expect_bytes(full, src[k].row_bytes);
                bulk_load(section, static_cast<const uint8_t *>(src[k].row0) + row * src[k].row_bytes, src[k].row_bytes, full);
            } else if (k < TXS) join_copy_from_before<TX>(section, full, src[k], row, rows);
            else                join_copy_from_before<TB>(section, full, src[k], row, rows);
        }
        mbar_arrive(full);                           // (with what was written by hand)
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
// A thread's eight columns from c on, neighbours or 32 apart, and whether they (VEC) or how many of them are there.
template <bool VEC> struct In { int n; };
template <> struct In<true> { bool n; };
template <bool VEC> __device__ __forceinline__ In<VEC> join_in(int c, int cols)
{
    if constexpr (VEC) return {c < cols};
    else return {min(max((cols - c + 31) >> 5, 0), 8)};
}
template <bool VEC> __device__ __forceinline__ In<VEC> operator&&(In<VEC> in, bool there)
{
    if constexpr (VEC) return {in.n && there};
    else return {there ? in.n : 0};
}
// They, of a row in a slot (zero where there are none).
template <typename T, bool VEC> __device__ __forceinline__ void ring_read(const uint8_t *row, int c, In<VEC> in, float (&v)[8])
{
    if (VEC) {
        Raw8<T> r;
        const uint4 *p = reinterpret_cast<const uint4 *>(row + c * (int)sizeof(T));
#pragma unroll
        for (int i = 0; i < Pieces<T>::n; ++i) r.w[i] = in.n ? p[i] : make_uint4(0, 0, 0, 0);
        unpack8(r, v);
    } else {
        const T *p = reinterpret_cast<const T *>(row) + c;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = e < in.n ? real_of(p[32 * e]) : 0.0f;
    }
}
// They, rounded to the type, to a row in memory; v is what the stored values stand for.  wide: fp32 rows start on 32-byte boundaries.
template <typename T, bool VEC> __device__ __forceinline__ void join_put(void *row0, int64_t at, In<VEC> in, int wide, float (&v)[8])
{
    T *const p = static_cast<T *>(row0) + at;
    if (VEC) {
        const Raw8<T> r = pack8<T>(v);
        unpack8(r, v);
        if (!row0 || !in.n) return;
        if (Pieces<T>::n == 2 && wide) put32(p, r.w[0], r.w[Pieces<T>::n - 1]);
        else {
#pragma unroll
            for (int i = 0; i < Pieces<T>::n; ++i) reinterpret_cast<uint4 *>(p)[i] = r.w[i];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const T t = real_to<T>(v[e]);
            if (row0 && e < in.n) p[32 * e] = t;
            v[e] = real_of(t);
        }
    }
}
// gate * w_post of them (where there are none, ones or zeros)
template <bool VEC> __device__ __forceinline__ void join_gains(const float *gate, const float *w_post, int64_t gate_at, int c, int cols, float (&v)[8])
{
    float w[8];
    if (VEC) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = 1.0f;
        if (c >= cols) return;
        if (gate) unpack8(load8(gate + gate_at + c, 8, true), v);
        if (!w_post) return;
        unpack8(load8(w_post + c, 8, true), w);
    } else {
        load_params<false>(gate, gate_at, c, cols, v);
        load_params<false>(w_post, 0, c, cols, w);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= w[e];
}

// ---- wide rows, from memory -------------------------------------------------------------------------------------------------
constexpr int kJoinWide = 4;                         // times eight columns a thread
#endif

// ================================================================= host side
struct JoinShape { int ch, threads; bool warp, vec; };
constexpr size_t kJoinMaxRing = 200 * 1024;         // of a block
// Bytes of a slot for each row that a block takes at once, as the kernel lays it out.
static inline size_t join_slot(const qbp_resnorm_desc *d, const JoinShape &s, int tensors)
{
    const uint32_t x = (uint32_t)(d->cols * dtype_size(d->x_dtype)), b = (uint32_t)(d->cols * dtype_size(d->b_dtype));
    return (size_t)(s.warp ? kJoinWarpRows : 1) * (size_t)tensors * (s.vec ? join_section<true>(x) + join_section<true>(b) : join_section<false>(x) + join_section<false>(b));
}
// Blocks that an SM has threads for (16 warps, which their registers allow; 8 backwards where a row is a warp's).
static inline int join_per_sm(const JoinShape &s, int tensors) { return s.ch > 2 ? 1 : std::max((s.warp && tensors == 2 ? 256 : 512) / s.threads, 1); }
// Slots of a block's ring (forward of one tensor of each type, backwards of two): three, but two where an SM's blocks would ask for more
// than 112 KB at a time (fp32 stream, bf16 blocks, us with three and two: 30000 x 2048 forward 136 and 123, backward 208 and 182; with less, 16384 x
// 4096 bf16 forward 93 and 114; one block an SM, 8192 x 8192 134 and 149).
static inline int join_slots(const qbp_resnorm_desc *d, const JoinShape &s, int tensors)
{
    if (tensors == 2 && s.ch != 1) return kJoinBackSlots;
    return join_per_sm(s, tensors) == 1 || 3 * join_slot(d, s, tensors) * (size_t)join_per_sm(s, tensors) <= 112 * 1024 ? kJoinSlots : kJoinSlots - 1;
}
static inline size_t join_ring(const qbp_resnorm_desc *d, const JoinShape &s, int tensors) { return (size_t)join_slots(d, s, tensors) * join_slot(d, s, tensors); }
// Forward a thread takes sixteen columns.  Backwards it takes eight up to 4096 columns: a row's values then stay in registers behind the
// exchange of its sums, and its slot is free at once (as first built 16384 x 4096 206 us, with sixteen 247; 2000 x 2048 bf16 28 and 37).  32
// (without a ring) beyond 8192 and where two slots find no room: backwards of fp32 alone from 6400 columns on, 8192 x 8192 1260 us (with
// bf16 blocks 217).
static inline JoinShape join_shape(const qbp_resnorm_desc *d, int tensors, bool vec)
{
    const int chunks = (int)((d->cols + 255) / 256);                 // a warp's eight columns a lane
    if (chunks <= 2) return {chunks, 32 * kJoinWarpRows, true, vec};
    const JoinShape s = tensors == 2 && chunks <= 16 ? JoinShape{1, 32 * chunks, false, vec} : JoinShape{2, 32 * ((chunks + 1) / 2), false, vec};
    if (s.threads <= 512 && join_ring(d, s, tensors) <= kJoinMaxRing) return s;
    return {4, 32 * ((chunks + 3) / 4), false, vec};
}

// Runs `call` with the kernel's compile-time choices.
#define QBP_FOR_JOIN(shape, backwards, CH, WARP, MAXT, call)                                                                  \
    do {                                                                                                                      \
        if ((shape).warp && (shape).ch == 1) { constexpr int CH = 1, MAXT = 256; constexpr bool WARP = true; call; }          \
        else if ((shape).warp) { constexpr int CH = 2, MAXT = 256; constexpr bool WARP = true; call; }                        \
        else if ((shape).ch == 1 || (!(backwards) && (shape).threads <= 256)) {                                               \
            constexpr int CH = (backwards) ? 1 : 2, MAXT = (backwards) ? 512 : 256; constexpr bool WARP = false; call;        \
        } else { constexpr int CH = 2, MAXT = 512; constexpr bool WARP = false; call; }                                       \
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

// Whether rows, columns and gate_rows are such that no count made of them overflows (2^48 elements at most).
static inline bool join_extents_ok(const qbp_resnorm_desc *d)
{
    return d->rows >= 0 && d->cols >= 0 && d->gate_rows >= 0 && d->cols <= kJoinMaxCols && d->rows <= ((int64_t)1 << 48) / std::max<int64_t>(d->cols, 1);
}
static inline int check_join(const qbp_resnorm_desc *d, const char *name, const void *b, const float *gate, const float *w_post, const float *w_pre)
{
    if (!d) return fail(QBP_ERR_INVALID_ARG, "%s: NULL descriptor", name);
    if (!dtype_ok(d->x_dtype) || !dtype_ok(d->b_dtype)) return fail(QBP_ERR_INVALID_ARG, "%s: dtypes %d and %d", name, d->x_dtype, d->b_dtype);
    if (d->rows < 0 || d->cols < 0 || d->gate_rows < 0) return fail(QBP_ERR_INVALID_ARG, "%s: rows %lld, cols %lld, gate_rows %lld", name, (long long)d->rows, (long long)d->cols, (long long)d->gate_rows);
    if (!join_extents_ok(d)) return fail(QBP_ERR_UNSUPPORTED_SHAPE, "%s: %lld rows of %lld columns, at most 2^48 elements in rows of %lld", name, (long long)d->rows, (long long)d->cols, (long long)kJoinMaxCols);
    if (!(d->eps >= 0.0f) || !(d->p >= 0.0f && d->p <= 1.0f) || std::isinf(d->eps)) return fail(QBP_ERR_INVALID_ARG, "%s: eps %g, p %g", name, (double)d->eps, (double)d->p);
    if (d->index_base % 8) return fail(QBP_ERR_INVALID_ARG, "%s: index_base %llu is not a multiple of 8", name, (unsigned long long)d->index_base);
    if (!b && d->rows > 0 && d->cols > 0 && (d->post || gate || d->p > 0.0f)) return fail(QBP_ERR_INVALID_ARG, "%s: a norm after, a gate or dropout without a block output", name);
    for (const float *w : {gate, w_post, w_pre})
        if (!aligned_to(w, 4)) return fail(QBP_ERR_INVALID_ARG, "%s: misaligned parameters", name);
    return QBP_OK;
}
// A call with nothing to do (a workspace that is there gets its status word cleared all the same).
static inline int join_empty(void *ws, size_t ws_bytes, cudaStream_t st)
{
    if (ws && aligned_to(ws, 4) && ws_bytes >= 4) QBP_CUDA_OK(cudaMemsetAsync(ws, 0, 4, st));
    return QBP_OK;
}
static inline bool real_ok(const void *p, int dtype) { return p && aligned_to(p, dtype_size(dtype)); }
// Rows that share a row of the gate: of those that there are, however many more a gate row is for.
static inline int64_t join_gate_rows(const qbp_resnorm_desc *d) { return std::max<int64_t>(d->gate_rows ? std::min(d->gate_rows, d->rows) : d->rows, 1); }

// How the rows are cut for a grid of at most `most` blocks: items of neighbouring rows of one gate.  Blocks take items in turn, and the time
// is that of the block with the most: items fill whole rounds of the grid, one of them or up to three more where that is less for the
// busiest block.  An item costs a row beside its own, backwards three and a half: the ring drains, and sums are left (16384 x 4096 in items of
// eight rows 148 and 267 us, of one row 255 and 800, of many 139 and 197).  Cut into so many that every block had at least one, 16 gates of 1024 rows
// were 160 items for 148 blocks, and twelve blocks had two (4096 columns, fp32 / bf16, us so and as here: backward 330 and 204, forward 204 and
// 140; 8 gates of 2048 backward 345 and 206, 100 of 164 rows 305 and 256).  Backwards (`sums`) the parts of a cut gate are added up by
// join_sum_kernel, whose blocks take about a row's time for 128 columns of a gate each, two to an SM: 949 gates of 8 rows of 1312 columns in fp32 are 65 us
// whole and 188 us in halves.
struct JoinCut { JoinItems it; int64_t blocks; };
static inline JoinCut join_cut(const qbp_resnorm_desc *d, const JoinShape &s, bool per_gate, int64_t most, int64_t few, bool sums)
{
    JoinCut c{};
    JoinItems &it = c.it;
    it.rows = d->rows; it.cols = d->cols;
    it.gate_rows = per_gate ? join_gate_rows(d) : std::max<int64_t>(d->rows, 1);
    it.gates = std::max<int64_t>((d->rows + it.gate_rows - 1) / it.gate_rows, 1);
    const auto parts = [](int64_t n, int64_t of) { return (n + of - 1) / of; };
    const int64_t at_once = s.warp ? kJoinWarpRows : 1;              // a block takes so many rows at a time
    const int64_t beside = sums ? 7 : 2;                             // (in half rows, as the cost and `adding`)
    const int64_t adding = sums && it.gates > 1 ? 2 * (it.gates * parts(d->cols, 128) / (2 * sm_count())) : 0;
    const int64_t last_gate = it.rows - (it.gates - 1) * it.gate_rows;         // its rows, maybe fewer than the others'
    const int64_t finest = parts(it.gate_rows, few * at_once);
    int64_t best = std::numeric_limits<int64_t>::max();
    const auto consider = [&](int64_t splits) {
        const int64_t rows = parts(it.gate_rows, std::min(std::max<int64_t>(splits, 1), finest)), whole = parts(it.gate_rows, rows);
        const int64_t cost = parts((it.gates - 1) * whole + parts(last_gate, rows), most) * (2 * parts(rows, at_once) + beside) + (whole > 1 ? adding : 0);
        if (cost < best) { best = cost; it.split_rows = rows; it.splits = whole; }
    };
    if (it.gates == 1) consider(most);                               // (more rounds only add to it)
    else
        for (int64_t rounds = parts(it.gates, most), end = rounds + 4, splits = 0; rounds < end && splits <= finest; ++rounds) {
            splits = rounds * most * it.gate_rows / it.rows;
            consider(splits);
            consider(splits - 1);                                    // (the last gate's may be one too many)
        }
    c.blocks = std::min(most, it.gates * it.splits);
    return c;
}
// Blocks of a wave, or as many of an SM's as their rings leave room for.
static inline int64_t join_blocks(const qbp_resnorm_desc *d, const JoinShape &s, int tensors)
{
    const int64_t room = s.ch > 2 ? 1 : (int64_t)(227 * 1024 / (join_ring(d, s, tensors) + 2048 + (s.warp && tensors == 2 ? 16384 : 0)));
    return (int64_t)sm_count() * std::max<int64_t>(std::min<int64_t>(join_per_sm(s, tensors), room), 1);
}

}  // namespace qbp
