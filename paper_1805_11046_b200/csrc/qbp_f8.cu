// 8-bit floating point with a scale for each block of 128: the quantisers, the product of a few output tiles on single CTAs,
// and the entry points.  The scales' layout is described in qbp_f8.cuh; the product of many tiles runs on CTA pairs (qbp_f8_pair.cu).
#include "qbp_f8.cuh"

#include <algorithm>

namespace qbp {

// ================================================================== quantisers
// A block takes one 128 x 128 tile: thread t holds the eight columns 8 (t % 16) of the rows t / 16 + 16 i in registers, so
// that x is read once for both copies.  A row's largest magnitude is found by the sixteen lanes that hold it, a column's by a
// warp's two rows and then across the warps in shared memory.  The maxima pass a NaN on; a block that is not finite gets a NaN for
// its inverse scale, and with it NaN codes.
constexpr int kQuantThreads = 256;
constexpr int kQuantPasses = 8;

enum { kF8Rows = 1, kF8Cols = 2, kF8Square = 4 };

// The scale byte of outer index `o` (0..127 of the tile's piece) and block `b`; behind the last block, the rest of its word.
__device__ __forceinline__ void put_scale(uint8_t *piece, int o, int b, bool last, uint32_t byte)
{
    uint8_t *at = piece + (o & 31) * 16 + (o >> 5) * 4;
    if (!last) at[b] = (uint8_t)byte;
    else {
        const uint32_t pad = 0x7F7F7F7Fu << (8 * b), word = (byte << (8 * b)) | (b < 3 ? pad << 8 : 0u);
        for (int k = b; k < 4; ++k) at[k] = (uint8_t)(word >> (8 * k));
    }
}

template <typename T, int FORMAT, int WHAT>
__global__ void __launch_bounds__(kQuantThreads, sizeof(T) == 2 ? 3 : 2)
f8_quantize_kernel(const T *__restrict__ x, int64_t rows, int64_t cols, int64_t ld, int vec, uint8_t *__restrict__ q_rows, uint8_t *__restrict__ s_rows,
                   uint8_t *__restrict__ q_cols, uint8_t *__restrict__ s_cols)
{
    __shared__ float s_amax[kQuantThreads / 32][kF8Block];
    __shared__ float s_inv[kF8Block];
    const int lane16 = threadIdx.x & 15, high = threadIdx.x >> 4, warp = threadIdx.x >> 5;
    const int64_t tile_c = blockIdx.x, tile_r = blockIdx.y, r0 = tile_r * kF8Block, c0 = tile_c * kF8Block + 8 * lane16;
    const int here = (int)min((int64_t)kF8Block, rows - r0);                        // rows of the tile
    const bool in = c0 < cols;                                                      // (cols is a multiple of 16: all eight or none)
    // the tile's pieces: of its rows (blocks along the columns) and of its columns
    const int64_t blocks_c = (cols + 127) >> 7, blocks_r = (rows + 127) >> 7;
    uint8_t *const p_rows = s_rows + (tile_r * ((blocks_c + 3) >> 2) + (tile_c >> 2)) * kF8Piece;
    uint8_t *const p_cols = s_cols + (tile_c * ((blocks_r + 3) >> 2) + (tile_r >> 2)) * kF8Piece;
    const int b_rows = (int)tile_c & 3, b_cols = (int)tile_r & 3;
    const bool last_c = tile_c == blocks_c - 1, last_r = tile_r == blocks_r - 1;
    const T *src = x + (r0 + high) * ld + c0;
    pdl_wait();
    Raw8<T> raw[kQuantPasses];
    if (vec) {
#pragma unroll
        for (int i = 0; i < kQuantPasses; ++i)
#pragma unroll
            for (int k = 0; k < (int)(sizeof(T) / 2); ++k)
                raw[i].w[k] = in && 16 * i + high < here ? __ldg(reinterpret_cast<const uint4 *>(src + 16 * i * ld) + k) : make_uint4(0, 0, 0, 0);
    } else {
#pragma unroll
        for (int i = 0; i < kQuantPasses; ++i) raw[i] = load8(in && 16 * i + high < here ? src + 16 * i * ld : x, in && 16 * i + high < here ? 8 : 0, false);
    }
    float col_max[8], row_max[kQuantPasses];
    if constexpr (sizeof(T) == 2) {
        // two elements to a word
        using Max = HalfMax<T>;
        uint32_t c[4] = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < kQuantPasses; ++i) {
            const uint4 w = raw[i].w[0];
            const uint32_t a[4] = {w.x & 0x7FFF7FFFu, w.y & 0x7FFF7FFFu, w.z & 0x7FFF7FFFu, w.w & 0x7FFF7FFFu};
            if (WHAT & kF8Cols) {
#pragma unroll
                for (int k = 0; k < 4; ++k) c[k] = Max::max2(c[k], a[k]);
            }
            if (WHAT & (kF8Rows | kF8Square)) {
                const uint32_t m = Max::max2(Max::max2(a[0], a[1]), Max::max2(a[2], a[3]));
                row_max[i] = Max::value(Max::max2(m, m >> 16), 0);
            }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) { col_max[2 * k] = Max::value(c[k], 0); col_max[2 * k + 1] = Max::value(c[k], 1); }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) col_max[e] = 0.0f;
#pragma unroll
        for (int i = 0; i < kQuantPasses; i += 2) {
            float v[8], u[8];
            unpack8(raw[i], v); unpack8(raw[i + 1], u);
            if (WHAT & (kF8Rows | kF8Square)) {
                row_max[i] = amax3(amax3(amax3(amax3(v[0], v[1], v[2]), v[3], v[4]), v[5], v[6]), v[7], 0.0f);
                row_max[i + 1] = amax3(amax3(amax3(amax3(u[0], u[1], u[2]), u[3], u[4]), u[5], u[6]), u[7], 0.0f);
            }
            if (WHAT & kF8Cols) {
#pragma unroll
                for (int e = 0; e < 8; ++e) col_max[e] = amax3(col_max[e], v[e], u[e]);
            }
        }
    }
    float col_inv[8], tile_inv = 1.0f;
    if (WHAT & kF8Cols) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            col_max[e] = amax3(col_max[e], __shfl_xor_sync(0xFFFFFFFFu, col_max[e], 16), 0.0f);
            if ((threadIdx.x & 16) == 0) s_amax[warp][8 * lane16 + e] = col_max[e];
        }
        __syncthreads();
        if (threadIdx.x < kF8Block) {
            float m = 0.0f;
#pragma unroll
            for (int w = 0; w < kQuantThreads / 32; w += 2) m = amax3(m, s_amax[w][threadIdx.x], s_amax[w + 1][threadIdx.x]);
            const uint32_t byte = f8_scale_byte<FORMAT>(m);                         // (127 for columns behind the last)
            s_inv[threadIdx.x] = f8_inverse(byte);
            put_scale(p_cols, threadIdx.x, b_cols, last_r, byte);
        }
        __syncthreads();
        const float4 a = *reinterpret_cast<const float4 *>(s_inv + 8 * lane16), b = *reinterpret_cast<const float4 *>(s_inv + 8 * lane16 + 4);
        col_inv[0] = a.x; col_inv[1] = a.y; col_inv[2] = a.z; col_inv[3] = a.w; col_inv[4] = b.x; col_inv[5] = b.y; col_inv[6] = b.z; col_inv[7] = b.w;
    }
    if (WHAT & kF8Square) {
        float m = 0.0f;
#pragma unroll
        for (int i = 0; i < kQuantPasses; i += 2) m = amax3(m, row_max[i], row_max[i + 1]);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m = amax3(m, __shfl_xor_sync(0xFFFFFFFFu, m, o), 0.0f);
        if ((threadIdx.x & 31) == 0) s_amax[warp][0] = m;
        __syncthreads();
        m = 0.0f;
#pragma unroll
        for (int w = 0; w < kQuantThreads / 32; w += 2) m = amax3(m, s_amax[w][0], s_amax[w + 1][0]);
        const uint32_t byte = f8_scale_byte<FORMAT>(m);
        tile_inv = f8_inverse(byte);
        if (threadIdx.x < kF8Block) {
            if (s_rows) put_scale(p_rows, threadIdx.x, b_rows, last_c, (int)threadIdx.x < here ? byte : 127u);
            if (s_cols) put_scale(p_cols, threadIdx.x, b_cols, last_r, tile_c * kF8Block + threadIdx.x < cols ? byte : 127u);
        }
    }
    float row_inv = 1.0f;                                     // of row 16 (lane16 / 2) + high
    if (WHAT & kF8Rows) {
        // The eight rows' maxima over the sixteen lanes, halving the rows a lane is concerned with at each exchange: lane 2 i ends with
        // row 16 i + high, and works out its scale alone.
        float a[4], b[2], m;
        const bool up8 = (lane16 & 8) != 0, up4 = (lane16 & 4) != 0, up2 = (lane16 & 2) != 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) a[j] = amax3(up8 ? row_max[j + 4] : row_max[j], __shfl_xor_sync(0xFFFFFFFFu, up8 ? row_max[j] : row_max[j + 4], 8), 0.0f);
#pragma unroll
        for (int j = 0; j < 2; ++j) b[j] = amax3(up4 ? a[j + 2] : a[j], __shfl_xor_sync(0xFFFFFFFFu, up4 ? a[j] : a[j + 2], 4), 0.0f);
        m = amax3(up2 ? b[1] : b[0], __shfl_xor_sync(0xFFFFFFFFu, up2 ? b[0] : b[1], 2), 0.0f);
        m = amax3(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1), 0.0f);
        const uint32_t byte = f8_scale_byte<FORMAT>(m);
        row_inv = f8_inverse(byte);
        if ((lane16 & 1) == 0) put_scale(p_rows, 8 * lane16 + high, b_rows, last_c, byte);         // (127 for rows behind the last)
    }
    uint8_t *d_rows = q_rows + (r0 + high) * cols + c0, *d_cols = q_cols + (r0 + high) * cols + c0;
#pragma unroll
    for (int i = 0; i < kQuantPasses; ++i) {
        float v[8], inv = tile_inv;
        unpack8(raw[i], v);
        if (WHAT & kF8Rows) inv = __shfl_sync(0xFFFFFFFFu, row_inv, (threadIdx.x & 16) | (2 * i));
        if (16 * i + high < here && in) {
            if (WHAT & (kF8Rows | kF8Square)) {
                float t[8];
#pragma unroll
                for (int e = 0; e < 8; e += 2) { t[e] = v[e]; t[e + 1] = v[e + 1]; mul2(t[e], t[e + 1], inv, inv); }
                *reinterpret_cast<uint2 *>(d_rows) = f8_codes8<FORMAT>(t);
            }
            if (WHAT & kF8Cols) {
#pragma unroll
                for (int e = 0; e < 8; e += 2) mul2(v[e], v[e + 1], col_inv[e], col_inv[e + 1]);
                *reinterpret_cast<uint2 *>(d_cols) = f8_codes8<FORMAT>(v);
            }
        }
        d_rows += 16 * cols; d_cols += 16 * cols;
    }
}

template <typename T, int FORMAT>
static void launch_f8_quantize_as(const T *x, int64_t rows, int64_t cols, int64_t ld, int what, uint8_t *q_rows, uint8_t *s_rows, uint8_t *q_cols,
                                  uint8_t *s_cols, cudaStream_t st)
{
    const dim3 grid((unsigned)f8_blocks(cols), (unsigned)f8_blocks(rows));
    const int vec = aligned16(x) && ld * sizeof(T) % 16 == 0 ? 1 : 0;
    auto *kernel = what == kF8Rows             ? f8_quantize_kernel<T, FORMAT, kF8Rows>
                   : what == kF8Cols           ? f8_quantize_kernel<T, FORMAT, kF8Cols>
                   : what == kF8Square         ? f8_quantize_kernel<T, FORMAT, kF8Square>
                                               : f8_quantize_kernel<T, FORMAT, kF8Rows | kF8Cols>;
    launch(kernel, grid, kQuantThreads, 0, st, x, rows, cols, ld, vec, q_rows, s_rows, q_cols, s_cols);
}

static int launch_f8_quantize(const void *x, int dtype, int64_t rows, int64_t cols, int64_t ld, int format, int what, uint8_t *q_rows,
                              uint8_t *s_rows, uint8_t *q_cols, uint8_t *s_cols, cudaStream_t st)
{
    QBP_TRACE_BEGIN(st);
    if (format == QBP_E4M3) QBP_FOR_DTYPE(dtype, T, (launch_f8_quantize_as<T, QBP_E4M3>((const T *)x, rows, cols, ld, what, q_rows, s_rows, q_cols, s_cols, st)));
    else                    QBP_FOR_DTYPE(dtype, T, (launch_f8_quantize_as<T, QBP_E5M2>((const T *)x, rows, cols, ld, what, q_rows, s_rows, q_cols, s_cols, st)));
    QBP_LAUNCH_OK("f8_quantize_kernel");
    return QBP_OK;
}

// ============================================================ the split product
// Few output tiles: a tile of 128 columns of the output by `bn` of its rows, its reduction split over the CTAs of a cluster.
// The columns' operand (a layer's weights) is the 128-row side of the MMA and the rows (tokens, 16 to 128 of them) its N
// side: a token or two then cost an N of 16 and not an M of 128, the accumulator's lanes are neighbouring outputs in memory,
// and the weights, all that counts when rows are few, are read once, by as many SMs as there are tiles times pieces of the
// reduction.  Each CTA of a cluster adds up a share of the rows, in the order of the pieces: the others write their fp32 partial
// sums of these rows into its shared memory (reading them there took a round trip a row: 128 x 1024 x 512 22.6 us with the launch).
//
// Roles: warp 0 loads by TMA, warp 1 copies scales to tensor memory and issues the MMAs, warps 2..9 take the accumulator out.
// Of a layer that serves up to eight rows (TX: their type), warps 2..9 first quantise the rows, each CTA its part of the reduction, straight into
// the stages, with the scales of one block at a time.
// Every wait is bounded.
constexpr int kSplitThreads = 320;
constexpr int kSplitMaxStages = 10;
constexpr uint32_t kSplitRelease = 2;            // stages released by one commit
constexpr int kSplitMaxParts = 8;
constexpr uint32_t kSplitSmem = 220u * 1024u;
constexpr uint32_t kSplitCols = 256;             // tensor memory: the accumulator in [0, 128), then sets of 4 columns of scales:
constexpr uint32_t kSplitSetU = 128, kSplitSetV = 144;
constexpr int kSplitSets = 4, kSplitBlockSets = 16;      // of U (and of V from memory), a set for four blocks; of V quantised here, for one
constexpr int64_t kSplitQuantise = 8;            // rows that every CTA quantises for itself, at most
constexpr size_t kSplitClusterSmem = 116u * 1024u;

struct F8SplitParams {
    CUtensorMap mapU, mapV;                      // U: the output's columns (operand B), V: its rows (operand A)
    const uint8_t *su, *sv;                      // their scales
    int64_t groups;                              // pieces of scales along the reduction
    const void *x; int64_t ld, K; int vec;       // the rows as real numbers, quantised here (no mapV, no sv)
    OperandLayout u, v;
    uint32_t idesc, stage_bytes;
    int bn, stages, k_blocks, parts;
    int64_t M, N;
    void *out; int dtype;
    int *status;
};

__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t address_in_cta(uint32_t smem_addr, uint32_t rank)
{
    uint32_t at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_addr), "r"(rank));
    return at;
}
__device__ __forceinline__ void store_in_cta(uint32_t cluster_addr, uint32_t v)
{
    asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(cluster_addr), "r"(v) : "memory");
}

// A warp's 16 rows of the accumulator (rows: those that exist) to the output, n: the lane's column.
template <typename T> __device__ __forceinline__ void split_put(void *out, int64_t m, int64_t N, int64_t n, int rows, const uint32_t (&r)[16])
{
    T *o = static_cast<T *>(out) + m * N + n;
    if (n < N) {
#pragma unroll
        for (int j = 0; j < 16; ++j, o += N)
            if (j < rows) *o = real_to<T>(__uint_as_float(r[j]));
    }
}
// The sums of a part's rows, `step` apart from row `first` on, added up over the parts and stored.
template <typename T> __device__ __forceinline__ void split_add(void *out, int64_t m, int64_t N, int64_t n, int first, int step, int rows, int parts, int share, const float *sums)
{
    T *o = static_cast<T *>(out) + (m + first) * N + n;
    if (n < N) {
#pragma unroll 2
        for (int j = first; j < rows; j += step, o += step * N) {
            float v[kSplitMaxParts];
#pragma unroll
            for (int q = 0; q < kSplitMaxParts; ++q) v[q] = q < parts ? sums[(q * share + j) * 128] : 0.0f;
            float t = 0.0f;
#pragma unroll
            for (int q = 0; q < kSplitMaxParts; ++q) t += v[q];
            *o = real_to<T>(t);
        }
    }
}

// Warps 2..9: the blocks kb0..kb1 of all rows (at most kSplitQuantise) to e4m3, into the stages as the product wants them: rows of 128 bytes,
// 16-byte pieces swizzled by the row, and each row's scale byte at its place in a piece.  A block is a warp's (with all warps on one
// block, one block after the other, a block took half a microsecond, nearly all of it latency), two rows at a time, sixteen lanes to a row, all
// rows' loads on their way at once.  No more warps than stages take part: a stage is then written at most a round after the warp's own last
// block, and the parity of its barrier tells whether that round is free; for a stage further ahead, the round before the last would pass for
// it.  False when a wait ran out.
template <typename T>
__device__ __forceinline__ bool split_quantise(const F8SplitParams &P, uint8_t *smem, uint64_t *full_bar, uint64_t *empty_bar, int kb0, int kb1)
{
    const int lane = threadIdx.x & 31, lane16 = lane & 15, high = lane >> 4;
    const int M = (int)P.M, warps = min(8, P.stages), me = (int)(threadIdx.x >> 5) - 2;
    uint32_t s = (uint32_t)me, ph = 1;
    for (int kb = kb0 + me; me < warps && kb < kb1; kb += warps) {
        const int64_t c = 128ll * kb + 8 * lane16;
        const T *x = static_cast<const T *>(P.x) + (c < P.K ? c : 0);
        const auto load = [&](int r) { return load8(x + (r < M ? r : 0) * P.ld, r < M && c < P.K ? 8 : 0, P.vec != 0); };
        Raw8<T> raw[kSplitQuantise / 2];
#pragma unroll
        for (int a = 0; a < (int)kSplitQuantise / 2; ++a) raw[a] = load(2 * a + high);
        if (!mbar_wait_warp(&empty_bar[s / kSplitRelease], ph)) return false;
        uint8_t *const sv = smem + (size_t)s * P.stage_bytes + P.u.tile_bytes, *const bytes = sv + P.v.tile_bytes + kF8Piece + (kb & 3);
#pragma unroll
        for (int a = 0; a < (int)kSplitQuantise / 2; ++a) {
            const int r = 2 * a + high;
            if (2 * a >= M) break;
            float v[8];
            unpack8(raw[a], v);
            float m = amax3(amax3(amax3(amax3(v[0], v[1], v[2]), v[3], v[4]), v[5], v[6]), v[7], 0.0f);
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) m = amax3(m, __shfl_xor_sync(0xFFFFFFFFu, m, o), 0.0f);
            const uint32_t byte = f8_scale_byte<QBP_E4M3>(m);
            const float inv = f8_inverse(byte);
            if (r < M) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = __fmul_rn(v[e], inv);
                *reinterpret_cast<uint2 *>(sv + r * 128 + (((lane16 >> 1) ^ (r & 7)) << 4) + (lane16 & 1) * 8) = f8_codes8<QBP_E4M3>(v);
                if (lane16 == 0) bytes[r * 16] = (uint8_t)byte;
            }
        }
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(&full_bar[s]);
        s += (uint32_t)warps;
        if (s >= (uint32_t)P.stages) { s -= (uint32_t)P.stages; ph ^= 1u; }
    }
    return true;
}

struct FromCodes {};
template <typename TX> struct SplitRows { static constexpr bool quantise = true; using type = TX; };
template <> struct SplitRows<FromCodes> { static constexpr bool quantise = false; using type = float; };

template <typename TX>
__global__ void __launch_bounds__(kSplitThreads, 2) f8_split_kernel(const __grid_constant__ F8SplitParams P)
{
    constexpr bool kQuantise = SplitRows<TX>::quantise;
    using T = typename SplitRows<TX>::type;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t full_bar[kSplitMaxStages], empty_bar[kSplitMaxStages / kSplitRelease], acc_full;
    __shared__ uint32_t tmem_slot;
    const uint32_t raw_addr = smem_u32(smem_raw);
    uint8_t *smem = smem_raw + ((1024u - (raw_addr & 1023u)) & 1023u);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int part = (int)cluster_rank();
    const int64_t n0 = (int64_t)(blockIdx.x / P.parts) * 128, m0 = (int64_t)blockIdx.y * P.bn;
    const int kb0 = (int)((int64_t)P.k_blocks * part / P.parts), kb1 = (int)((int64_t)P.k_blocks * (part + 1) / P.parts);

    if (threadIdx.x == 0) {
        for (int s = 0; s < P.stages; ++s) mbar_init(&full_bar[s], kQuantise ? 2 : 1);
        for (int g = 0; g < P.stages / (int)kSplitRelease; ++g) mbar_init(&empty_bar[g], 1);
        mbar_init(&acc_full, 1);
        mbar_fence_init();
        tma_prefetch_desc(&P.mapU);
        if (!kQuantise) tma_prefetch_desc(&P.mapV);
    }
    if (warp == 1) { tmem_alloc(&tmem_slot, kSplitCols); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    bool timed_out = false;
    if (P.parts > 1) cluster_arrive();               // (the others' wait for it: this CTA runs, its memory can be written)
    pdl_wait();
    // The status word is cleared here and not by a launch of its own: a wait gives up a second after it began, long after the
    // first block of a grid has started.
    if (threadIdx.x == 0 && blockIdx.x == 0 && blockIdx.y == 0) *P.status = 0;

    if (warp == 0) {
        // (the whole warp in step, an elected lane issues, as in the pair kernel)
        uint32_t s = 0, ph = 1, in_group = 0, group = 0;
        const bool u_k = P.u.major == 0, v_k = P.v.major == 0;
        for (int kb = kb0; kb < kb1; ++kb) {
            if (in_group == 0 && !mbar_wait_uniform(&empty_bar[group], ph)) { timed_out = true; break; }
            if (++in_group == kSplitRelease) { in_group = 0; ++group; }
            uint8_t *su = smem + (size_t)s * P.stage_bytes, *sv = su + P.u.tile_bytes, *scales = sv + P.v.tile_bytes;
            const bool with_scales = kb == kb0 || (kb & 3) == 0;
            const int k0 = kb * 128;
            if (elect_one()) {
                mbar_expect_tx(&full_bar[s], P.u.tile_bytes + (kQuantise ? 0u : P.v.tile_bytes) + (with_scales ? (kQuantise ? 1u : 2u) * kF8Piece : 0u));
                tma_load_2d(su, &P.mapU, &full_bar[s], u_k ? k0 : (int)n0, u_k ? (int)n0 : k0);
                if (!kQuantise) tma_load_2d(sv, &P.mapV, &full_bar[s], v_k ? k0 : (int)m0, v_k ? (int)m0 : k0);
                if (with_scales) {
                    bulk_load(scales, P.su + ((n0 >> 7) * P.groups + (kb >> 2)) * kF8Piece, kF8Piece, &full_bar[s]);
                    if (!kQuantise) bulk_load(scales + kF8Piece, P.sv + ((m0 >> 7) * P.groups + (kb >> 2)) * kF8Piece, kF8Piece, &full_bar[s]);
                }
            }
            __syncwarp();
            if (++s == (uint32_t)P.stages) { s = 0; ph ^= 1u; group = 0; }
        }
    } else if (warp == 1) {
        uint32_t s = 0, ph = 0, set = kSplitSets - 1, vset = kSplitBlockSets - 1, in_group = 0, group = 0;
        bool ready = false;
        for (int kb = kb0; kb < kb1; ++kb) {
            if (!__all_sync(0xffffffffu, ready) && !mbar_wait_uniform(&full_bar[s], ph)) { timed_out = true; break; }
            tc_fence_after();
            const uint32_t su = smem_u32(smem) + s * P.stage_bytes, sv = su + P.u.tile_bytes, scales = sv + P.v.tile_bytes;
            if (++s == (uint32_t)P.stages) { s = 0; ph ^= 1u; }
            ready = mbar_test(&full_bar[s], ph);
            // (a set's last readers, the MMAs of at least 4 (kSplitSets - 1) + 1 blocks ago, or kSplitBlockSets, are done: the stage of a
            // later block than theirs has been filled again, at most kSplitMaxStages + kSplitRelease blocks ago)
            const bool with_scales = kb == kb0 || (kb & 3) == 0;
            if (with_scales) set = set + 1 == kSplitSets ? 0u : set + 1;
            if (kQuantise) vset = vset + 1 == kSplitBlockSets ? 0u : vset + 1;
            const uint32_t t_su = tmem + kSplitSetU + 4u * set, t_sv = tmem + kSplitSetV + 4u * (kQuantise ? vset : set);
            if ((kQuantise || with_scales) && elect_one()) {
                if (with_scales) copy_piece(t_su, piece_desc(scales));
                copy_piece(t_sv, piece_desc(scales + kF8Piece));
            }
            const uint32_t id = (uint32_t)(kb & 3), idesc = P.idesc | (id << 4) | (id << 29);
            const uint32_t u_lo = ((su >> 4) & 0x3FFFu) | P.u.desc_lo, v_lo = ((sv >> 4) & 0x3FFFu) | P.v.desc_lo;
            if (elect_one()) {
#pragma unroll
                for (uint32_t kk = 0; kk < 4; ++kk)
                    mma_f8(tmem, ((uint64_t)P.u.desc_hi << 32) | (uint64_t)(u_lo + kk * P.u.kstep),
                           ((uint64_t)P.v.desc_hi << 32) | (uint64_t)(v_lo + kk * P.v.kstep), idesc, t_su, t_sv, kb == kb0 && kk == 0 ? 0u : 1u);
            }
            if (++in_group == kSplitRelease) {
                if (elect_one()) mma_commit(&empty_bar[group]);
                in_group = 0;
                if (++group * kSplitRelease == (uint32_t)P.stages) group = 0;
            }
        }
        if (!timed_out && elect_one()) mma_commit(&acc_full);
        __syncwarp();
    }
    // (bn and the parts are powers of two)
    const int quad = warp & 3, half = (warp - 2) >> 2, log_share = __ffs(P.bn) - __ffs(P.parts), share = 1 << log_share;       // rows that a part adds up
    const int64_t n = n0 + 32 * quad + lane;
    float *const sums = reinterpret_cast<float *>(smem + (size_t)P.stages * P.stage_bytes) + 32 * quad + lane;                // [parts][share][128]
    if (warp >= 2) {
        if (kQuantise) timed_out = !split_quantise<T>(P, smem, full_bar, empty_bar, kb0, kb1);
        if (!timed_out && !mbar_wait_warp(&acc_full, 0)) timed_out = true;
        tc_fence_after();
    }
    if (P.parts > 1) { __syncwarp(); cluster_wait(); }
    if (warp >= 2) {
        for (int c = 16 * half; c < P.bn && m0 + c < P.M && !timed_out; c += 32) {
            uint32_t r[16];
            tmem_ld_32x16(tmem + ((uint32_t)(32 * quad) << 16) + (uint32_t)c, r);
            tmem_ld_wait();
            const int rows = (int)min((int64_t)16, P.M - m0 - c);
            if (P.parts > 1) {
                const uint32_t mine = smem_u32(sums) + ((uint32_t)part << (9 + log_share));
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    if (j < rows) store_in_cta(address_in_cta(mine + (uint32_t)(((c + j) & (share - 1)) << 9), (uint32_t)((c + j) >> log_share)), r[j]);
            } else {
                if (P.dtype == QBP_F32) split_put<float>(P.out, m0 + c, P.N, n, rows, r);
                else if (P.dtype == QBP_BF16) split_put<__nv_bfloat16>(P.out, m0 + c, P.N, n, rows, r);
                else split_put<__half>(P.out, m0 + c, P.N, n, rows, r);
            }
        }
    }
    if (timed_out) { raise_timeout(P.status); __nanosleep(1000000); }
    tc_fence_before();
    __syncthreads();
    if (P.parts > 1) {
        cluster_arrive();
        cluster_wait();                                               // every part's sums are here; nobody writes behind this
        if (warp >= 2) {
            const int64_t m = m0 + part * share;
            const int rows = (int)max((int64_t)0, min((int64_t)share, P.M - m));
            if (P.dtype == QBP_F32) split_add<float>(P.out, m, P.N, n, half, 2, rows, P.parts, share, sums);
            else if (P.dtype == QBP_BF16) split_add<__nv_bfloat16>(P.out, m, P.N, n, half, 2, rows, P.parts, share, sums);
            else split_add<__half>(P.out, m, P.N, n, half, 2, rows, P.parts, share, sums);
        }
        __syncwarp();
    }
    if (warp == 1) { __syncwarp(); tmem_dealloc(tmem, kSplitCols); }
}

// A launch in clusters of `cluster` blocks, otherwise as launch().
template <typename... P, typename... A>
static void launch_clusters(void (*kernel)(P...), dim3 grid, unsigned cluster, unsigned threads, size_t smem, cudaStream_t st, A &&...args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid; cfg.blockDim = dim3(threads); cfg.dynamicSmemBytes = smem; cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = cluster; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = trace_is_on() ? 1 : 2;
    (void)cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}

// Clusters of `parts` CTAs that run at the same time, one CTA an SM (a cluster's SMs are of one GPC, whose number is no multiple of
// eight: of 16 clusters of eight some wait for the others).  Asked once per device.
static int split_clusters(int parts)
{
    static PerDeviceOnce asked[4];
    static int found[4][kMaxDevices];
    const int k = parts == 2 ? 1 : parts == 4 ? 2 : 3;
    int dev = -1;
    if (asked[k].pending(&dev)) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)(parts * 256)); cfg.blockDim = dim3(kSplitThreads); cfg.dynamicSmemBytes = kSplitSmem;
        cudaLaunchAttribute attr;
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = (unsigned)parts; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = 1;
        cfg.attrs = &attr; cfg.numAttrs = 1;
        int n = 0;
        // (asked before the first launch, which opts in to this much shared memory too)
        if (cudaFuncSetAttribute(f8_split_kernel<FromCodes>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSplitSmem) != cudaSuccess ||
            cudaOccupancyMaxActiveClusters(&n, f8_split_kernel<FromCodes>, &cfg) != cudaSuccess) { cudaGetLastError(); n = sm_count() / parts * 3 / 4; }
        if (dev < 0) return n;
        found[k][dev] = n;
        asked[k].mark(dev);
    }
    return found[k][dev];
}

// Rows as real numbers, to be quantised on the way (x NULL: codes and scales are there).
struct SplitInput { const void *x; int64_t ld; };

// How a product is cut: tiles of 128 by bn outputs, each in `parts`, with rings of `stages`.
struct SplitShape { int bn, k_blocks, parts, stages; int64_t tiles_n, tiles_m; uint32_t stage_bytes, sums_bytes; };
static SplitShape split_shape(const F8Product &p)
{
    SplitShape P{};
    P.bn = p.transA || p.M > 64 ? 128 : p.M > 32 ? 64 : p.M > 16 ? 32 : 16;
    P.k_blocks = (int)f8_blocks(p.K);
    P.tiles_n = f8_blocks(p.N); P.tiles_m = (p.M + P.bn - 1) / P.bn;
    // Parts: as many as run at the same time, where they save more blocks of 0.25 us than adding up the tile's rows costs (one call of
    // many in a row, one part and the best, us: 1 x 4096 x 4096 12.7 and 7.9 (four), 64 x 1024 x 1024 5.9 and 5.3 (eight), 128 x 1024 x
    // 1024 6.4 and 6.7 (eight), 512 x 2048 x 4096 14.3 and 14.1 (two), x 8192 23.9 and 20.6).
    P.parts = 1;
    while (P.parts < kSplitMaxParts && 2 * P.parts <= P.k_blocks && P.tiles_n * P.tiles_m <= split_clusters(2 * P.parts)) P.parts *= 2;
    if (P.k_blocks - (P.k_blocks + P.parts - 1) / P.parts <= 2 + P.bn / 16 * (P.parts == 2 ? 3 : 1)) P.parts = 1;
    P.stage_bytes = (uint32_t)align_up(128u * (128u + (uint32_t)P.bn) + 2u * kF8Piece, 1024);
    P.sums_bytes = P.parts > 1 ? (uint32_t)P.bn * 512u : 0u;
    P.stages = (int)std::min<int64_t>(kSplitMaxStages, (kSplitSmem - 1024 - P.sums_bytes) / P.stage_bytes);
    // more than a wave: two CTAs an SM, one's loads beside the other's epilogue
    if (P.tiles_n * P.tiles_m > sm_count()) P.stages = std::min<int>(P.stages, (int)((kSplitSmem / 2 - 2048) / P.stage_bytes));
    P.stages = std::min(P.stages, std::max(2, (P.k_blocks + P.parts - 1) / P.parts + 1));
    P.stages -= P.stages % (int)kSplitRelease;
    return P;
}

// Whether every CTA quantises the rows for itself, each warp some blocks one after the other, or a launch before does (one call of many in
// a row, on the way and apart, us: 1 x 1024 x 1024 5.8 and 6.6, 2 x 32768 x 4096 26.1 and 27.3, 4 x 32768 x 4096 29.9 and 27.3, 4 x 8192 x 8192 18.4
// and 19.0, 8 x 8192 x 8192 24.3 and 19.1, 8 x 4096 x 4096 9.5 and 9.4, 8 x 2048 x 8192 13.6 and 11.2, 16 x 4096 x 4096 11.0 and 9.5; a launch less is
// 2.4 of the host's where it is the bound).
static bool split_quantises(const F8Product &p)
{
    if (p.M > kSplitQuantise) return false;
    const SplitShape s = split_shape(p);
    const int blocks = (s.k_blocks + s.parts - 1) / s.parts, warps = std::min(8, s.stages), rounds = (blocks + warps - 1) / warps;
    return p.M * p.M * rounds <= 64;
}

static int launch_f8_split(const F8Product &p, const SplitInput &in, cudaStream_t st)
{
    F8SplitParams P{};
    int rc;
    static PerDeviceOnce configured;
    QBP_SMEM_OPT_IN(configured, f8_split_kernel<FromCodes>, kSplitSmem);
    const SplitShape s = split_shape(p);
    P.bn = s.bn; P.k_blocks = s.k_blocks; P.parts = s.parts; P.stages = s.stages; P.stage_bytes = s.stage_bytes;
    if (p.transB) { P.u = layout_kmajor(128, 128);        rc = make_map_2d(&P.mapU, p.B, p.N, p.K, 128, 128); }
    else          { P.u = layout_mnmajor(128, 128, 1, 0); rc = make_map_2d(&P.mapU, p.B, p.K, p.N, 128, 128); }
    if (rc) return rc;
    if (p.transA) P.v = layout_mnmajor(128, 128, 1, 0);
    else          P.v = layout_kmajor((uint32_t)P.bn, 128);
    P.idesc = make_idesc_f8(p.formatB, p.formatA, P.u.major, P.v.major, 128, (uint32_t)P.bn);
    static_assert(kSplitMaxStages + (int)kSplitRelease <= 4 * kSplitSets - 3 && kSplitMaxStages + (int)kSplitRelease < kSplitBlockSets &&
                  kSplitSetU + 4 * kSplitSets <= kSplitSetV && kSplitSetV + 4 * kSplitBlockSets <= kSplitCols, "a set of scales is written again while MMAs may read it");
    // A cluster's CTA has an SM to itself, as the pair kernels' have: where CTAs of two clusters shared one with a third that waits for their
    // tensor memory, while their peers wait for the third's on another SM, none would end.
    const size_t smem = std::max<size_t>(1024 + (size_t)P.stages * P.stage_bytes + s.sums_bytes, P.parts > 1 ? kSplitClusterSmem : 0);
    P.M = p.M; P.N = p.N; P.out = p.out; P.dtype = p.dtype; P.status = p.status;
    P.su = p.sB; P.groups = f8_groups(p.K);
    const dim3 grid((unsigned)(s.tiles_n * P.parts), (unsigned)s.tiles_m);
    if (in.x) {
        P.x = in.x; P.ld = in.ld; P.K = p.K;
        P.vec = aligned16(in.x) && in.ld * (int64_t)dtype_size(p.dtype) % 16 == 0 ? 1 : 0;
        QBP_TRACE_BEGIN(st);
        QBP_FOR_DTYPE(p.dtype, T, {
            static PerDeviceOnce once;
            QBP_SMEM_OPT_IN(once, f8_split_kernel<T>, kSplitSmem);
            launch_clusters(f8_split_kernel<T>, grid, (unsigned)P.parts, kSplitThreads, smem, st, P);
        });
        QBP_LAUNCH_OK("f8_split_kernel<quantise>");
        return QBP_OK;
    }
    P.sv = p.sA;
    if ((rc = p.transA ? make_map_2d(&P.mapV, p.A, p.K, p.M, 128, 128) : make_map_2d(&P.mapV, p.A, p.M, p.K, (uint32_t)P.bn, 128))) return rc;
    QBP_TRACE_BEGIN(st);
    launch_clusters(f8_split_kernel<FromCodes>, grid, (unsigned)P.parts, kSplitThreads, smem, st, P);
    QBP_LAUNCH_OK("f8_split_kernel");
    return QBP_OK;
}

// ================================================================= entry points
constexpr int64_t kF8MaxExtent = (int64_t)1 << 30;                  // TMA coordinates and the grid are 32-bit
constexpr int64_t kF8MaxRows = 65535 * 128;                         // the grid's second extent

static int check_quantize(const char *name, const void *x, int dtype, int64_t rows, int64_t cols, int64_t ld, int format)
{
    if (!dtype_ok(dtype)) return fail(QBP_ERR_INVALID_ARG, "%s: dtype %d", name, dtype);
    if (format != QBP_E4M3 && format != QBP_E5M2) return fail(QBP_ERR_INVALID_ARG, "%s: format %d", name, format);
    if (rows < 0 || cols < 0 || ld < cols) return fail(QBP_ERR_INVALID_ARG, "%s: rows %lld, cols %lld, ld %lld", name, (long long)rows, (long long)cols, (long long)ld);
    if (cols % 16) return fail(QBP_ERR_UNSUPPORTED_SHAPE, "%s: cols %lld is not a multiple of 16", name, (long long)cols);
    if (rows > kF8MaxRows || cols > kF8MaxExtent) return fail(QBP_ERR_UNSUPPORTED_SHAPE, "%s: %lld x %lld", name, (long long)rows, (long long)cols);
    if (rows == 0 || cols == 0) return QBP_OK;
    if (!x || !aligned_to(x, dtype_size(dtype))) return fail(QBP_ERR_INVALID_ARG, "%s: x is NULL or misaligned", name);
    return QBP_OK;
}

extern "C" __attribute__((visibility("default"))) size_t qbp_f8_scale_bytes(int64_t outer, int64_t reduction)
{
    if (outer <= 0 || reduction <= 0) return 0;
    return (size_t)(f8_blocks(outer) * f8_groups(reduction)) * kF8Piece;
}

extern "C" __attribute__((visibility("default"))) int qbp_quantize_f8(const void *x, int dtype, int64_t rows, int64_t cols, int64_t ld, int format,
                                                                      uint8_t *q_rows, uint8_t *s_rows, uint8_t *q_cols, uint8_t *s_cols, void *stream)
{
    int rc = check_quantize("quantize_f8", x, dtype, rows, cols, ld, format);
    if (rc || rows == 0 || cols == 0) return rc;
    if (!q_rows != !s_rows || !q_cols != !s_cols || (!q_rows && !q_cols)) return fail(QBP_ERR_INVALID_ARG, "quantize_f8: a copy needs both its codes and its scales");
    if (!aligned16(q_rows) || !aligned16(s_rows) || !aligned16(q_cols) || !aligned16(s_cols)) return fail(QBP_ERR_INVALID_ARG, "quantize_f8: codes and scales start on 16-byte boundaries");
    return launch_f8_quantize(x, dtype, rows, cols, ld, format, (q_rows ? kF8Rows : 0) | (q_cols ? kF8Cols : 0), q_rows, s_rows, q_cols, s_cols, (cudaStream_t)stream);
}

extern "C" __attribute__((visibility("default"))) int qbp_quantize_f8_square(const void *x, int dtype, int64_t rows, int64_t cols, int64_t ld, int format,
                                                                             uint8_t *q, uint8_t *s_rows, uint8_t *s_cols, void *stream)
{
    int rc = check_quantize("quantize_f8_square", x, dtype, rows, cols, ld, format);
    if (rc || rows == 0 || cols == 0) return rc;
    if (!q || (!s_rows && !s_cols)) return fail(QBP_ERR_INVALID_ARG, "quantize_f8_square: NULL codes, or neither table of scales");
    if (!aligned16(q) || !aligned16(s_rows) || !aligned16(s_cols)) return fail(QBP_ERR_INVALID_ARG, "quantize_f8_square: codes and scales start on 16-byte boundaries");
    return launch_f8_quantize(x, dtype, rows, cols, ld, format, kF8Square, q, s_rows, nullptr, s_cols, (cudaStream_t)stream);
}

// Whether the product runs on single CTAs.
// One wave of tiles of 128 on single CTAs against tiles of 256 rows on pairs (one call of many in a row, split and pair, us): 64 x 4096 x
// 8192 15.7 and 27.3, 512 x 4096 x 512 9.9 and 11.5, 1111 x 2048 x 8192 27.6 and 31.0; two waves: 512 x 8192 x 2048 26.3 and 17.4.
// Few rows are always theirs, whose half of the MMA is as narrow as they are: 1 x 32768 x 4096 28.6 and 44.1.
static bool one_wave(const F8Product &p)
{
    const int64_t rows = p.transA || p.M > 64 ? 128 : 64;
    return f8_blocks(p.N) * ((p.M + rows - 1) / rows) <= sm_count() || (!p.transA && p.M <= 128);
}
static int run_product(const F8Product &p, cudaStream_t st) { return one_wave(p) ? launch_f8_split(p, SplitInput{nullptr, 0}, st) : launch_f8_pair(p, st); }

static int check_product(const F8Product &p, const char *name)
{
    if (!dtype_ok(p.dtype)) return fail(QBP_ERR_INVALID_ARG, "%s: dtype %d", name, p.dtype);
    for (int f : {p.formatA, p.formatB})
        if (f != QBP_E4M3 && f != QBP_E5M2) return fail(QBP_ERR_INVALID_ARG, "%s: format %d", name, f);
    if (p.M < 0 || p.N < 0 || p.K < 0) return fail(QBP_ERR_INVALID_ARG, "%s: M %lld, N %lld, K %lld", name, (long long)p.M, (long long)p.N, (long long)p.K);
    const int64_t inner_a = p.transA ? p.M : p.K, inner_b = p.transB ? p.K : p.N;
    if (inner_a % 16 || inner_b % 16)
        return fail(QBP_ERR_UNSUPPORTED_SHAPE, "%s: the operands' innermost extents %lld and %lld are not multiples of 16", name, (long long)inner_a, (long long)inner_b);
    if (p.M > kF8MaxExtent || p.N > kF8MaxExtent || p.K > kF8MaxExtent || p.M > kF8MaxRows)
        return fail(QBP_ERR_UNSUPPORTED_SHAPE, "%s: %lld x %lld x %lld", name, (long long)p.M, (long long)p.N, (long long)p.K);
    return QBP_OK;
}

extern "C" __attribute__((visibility("default"))) size_t qbp_gemm_f8_workspace_bytes(int64_t M, int64_t N, int64_t K)
{
    (void)M; (void)N; (void)K;
    return 256;                                                      // the status word
}

extern "C" __attribute__((visibility("default"))) int qbp_gemm_f8(int transA, int transB, int64_t M, int64_t N, int64_t K, int formatA, const uint8_t *A,
                                                                  const uint8_t *sA, int formatB, const uint8_t *B, const uint8_t *sB, int out_dtype,
                                                                  void *out, void *ws, size_t ws_bytes, void *stream)
{
    cudaStream_t st = (cudaStream_t)stream;
    F8Product p{transA, transB, M, N, K, formatA, formatB, A, sA, B, sB, out, out_dtype, static_cast<int *>(ws)};
    int rc = check_product(p, "gemm_f8");
    if (rc) return rc;
    if (!ws || !aligned_to(ws, 256) || ws_bytes < qbp_gemm_f8_workspace_bytes(M, N, K))
        return fail(QBP_ERR_WORKSPACE, "gemm_f8: workspace NULL, misaligned or smaller than %zu bytes", qbp_gemm_f8_workspace_bytes(M, N, K));
    if (M == 0 || N == 0) { QBP_CUDA_OK(cudaMemsetAsync(ws, 0, 4, st)); return QBP_OK; }
    if (!out || !aligned_to(out, dtype_size(out_dtype))) return fail(QBP_ERR_INVALID_ARG, "gemm_f8: out is NULL or misaligned");
    if (K == 0) {
        QBP_CUDA_OK(cudaMemsetAsync(ws, 0, 4, st));
        QBP_CUDA_OK(cudaMemsetAsync(out, 0, (size_t)M * (size_t)N * dtype_size(out_dtype), st));
        return QBP_OK;
    }
    for (const void *t : {(const void *)A, (const void *)sA, (const void *)B, (const void *)sB})
        if (!t || !aligned16(t)) return fail(QBP_ERR_INVALID_ARG, "gemm_f8: an operand or its scales are NULL or not on a 16-byte boundary");
    return run_product(p, st);
}

extern "C" __attribute__((visibility("default"))) size_t qbp_linear_f8_workspace_bytes(int64_t M, int64_t N, int64_t K)
{
    (void)N;
    if (M <= 0 || K <= 0) return 256;
    return 256 + align_up((size_t)M * (size_t)K, 256) + align_up(qbp_f8_scale_bytes(M, K), 256);
}

extern "C" __attribute__((visibility("default"))) int qbp_linear_f8(const void *x, int dtype, int64_t ld, int64_t M, int64_t N, int64_t K, int w_format,
                                                                    const uint8_t *w, const uint8_t *sw, void *y, void *ws, size_t ws_bytes, void *stream)
{
    cudaStream_t st = (cudaStream_t)stream;
    F8Product p{0, 1, M, N, K, QBP_E4M3, w_format, nullptr, nullptr, w, sw, y, dtype, static_cast<int *>(ws)};
    int rc = check_product(p, "linear_f8");
    if (rc) return rc;
    if ((rc = check_quantize("linear_f8", x, dtype, M, K, ld, QBP_E4M3))) return rc;
    if (!ws || !aligned_to(ws, 256) || ws_bytes < qbp_linear_f8_workspace_bytes(M, N, K))
        return fail(QBP_ERR_WORKSPACE, "linear_f8: workspace NULL, misaligned or smaller than %zu bytes", qbp_linear_f8_workspace_bytes(M, N, K));
    if (M == 0 || N == 0) { QBP_CUDA_OK(cudaMemsetAsync(ws, 0, 4, st)); return QBP_OK; }
    if (!y || !aligned_to(y, dtype_size(dtype))) return fail(QBP_ERR_INVALID_ARG, "linear_f8: y is NULL or misaligned");
    if (K == 0) {
        QBP_CUDA_OK(cudaMemsetAsync(ws, 0, 4, st));
        QBP_CUDA_OK(cudaMemsetAsync(y, 0, (size_t)M * (size_t)N * dtype_size(dtype), st));
        return QBP_OK;
    }
    if (!w || !sw || !aligned16(w) || !aligned16(sw)) return fail(QBP_ERR_INVALID_ARG, "linear_f8: the weights or their scales are NULL or not on a 16-byte boundary");
    if (split_quantises(p)) return launch_f8_split(p, SplitInput{x, ld}, st);
    WsCarver c(ws, ws_bytes);
    c.take<int>(1);
    uint8_t *q = c.take<uint8_t>((size_t)M * (size_t)K), *s = c.take<uint8_t>(qbp_f8_scale_bytes(M, K));
    if ((rc = launch_f8_quantize(x, dtype, M, K, ld, QBP_E4M3, kF8Rows, q, s, nullptr, nullptr, st))) return rc;
    p.A = q; p.sA = s;
    return run_product(p, st);
}

}  // namespace qbp
