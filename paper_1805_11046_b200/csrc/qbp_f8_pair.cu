// The product of 8-bit floating-point codes with a scale for each block of 128, many output tiles: on CTA pairs,
// tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.
//
// Two CTAs of a cluster compute one 256 x bn output tile (bn 256 or 128): CTA r holds 128 of its rows of A and bn / 2 of its
// columns of B in shared memory, and the accumulator of its 128 rows in its tensor memory; one thread of the first CTA issues
// every MMA.  The scales go with every fourth stage (a piece covers four blocks of the reduction): each CTA's 128 of A and all
// bn of B, which both SMs' tensor cores need, and a tcgen05.cp ahead of the stage's MMAs moves them to tensor memory.  The
// scales cost the tensor pipe nothing then: they are powers of two and the MMA applies them.
//
// Tensor memory (512 columns).  Two accumulators of 256 columns would leave none for the scales, so of bn = 256 the second begins
// at column 192: the last 64 columns of one are the first 64 of the other.  The epilogue of a tile takes these out first, and
// the next tile's MMAs wait for no more than that.  [448, 508) then holds five sets of scales of 12 columns.
//
// A set is written again without a wait of its own.  Of bn = 256 a tile starts when all MMAs before it are done (its accumulator shares
// columns with the last one), and within a tile five sets are at least 17 blocks apart; of bn = 128 a tile starts when all but the last tile's
// are done, and eight sets are more than 24 blocks apart within two tiles.  That is more than a ring and a release group: the stage of a
// block has been filled, so the MMAs of the block that had it before are done.
//
// The issuing thread's own time counts: a block's four MMAs are 512 cycles, and with a commit for every block, a wait for its stage that began
// when its MMAs were due and a barrier for the scales' sets the loop took 740.  Stages are released two at a time, and a stage's barrier
// is asked while the MMAs before it are being issued.
//
// Roles per CTA: warp 0 loads by TMA, warp 1 (first CTA) issues copies of scales and MMAs, warps 2..9 drain the accumulator
// and store.  Every wait is bounded; on expiry the CTA raises the status word and leaves through the normal exit.  No TMA load
// here uses cluster multicast.
#include "qbp_f8.cuh"
#include "qbp_pair.cuh"

#include <algorithm>

namespace qbp {

constexpr int kFpThreads = 320;
constexpr int kFpEpiWarps = 8;
constexpr int kFpMaxStages = 8;
constexpr int kFpGroupM = 8;                     // tiles walk down eight tile rows before moving one column right
constexpr uint32_t kFpRelease = 2;               // stages released by one commit
constexpr uint32_t kFpSlab = 32 * 64;            // staging of a warp: 32 rows of 64 bytes
constexpr uint32_t kFpSmem = 225u * 1024u;

struct F8PairParams {
    CUtensorMap mapA, mapB, mapSA, mapSB, mapC;
    OperandLayout a, b;                          // per-CTA halves: A 128 rows, B bn / 2 columns, 128 reduction bytes
    uint32_t idesc, stage_bytes;
    int bn, stages, k_blocks;
    uint32_t buf1, set_col, set_cols, sets;      // first column of the second accumulator, of the scales; columns of a set
    int overlap;                                 // the accumulators share 64 columns
    int tiles_m, tiles_n, tiles_total, pairs;
    FastDiv d_group;
    int64_t M, N;
    void *out; int dtype, tma_out;
    int *status;
};

__device__ __forceinline__ void tma_load_3d_pair(void *dst, const void *map, uint32_t bar_cluster_addr, int x, int y, int z)
{
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
        ::"r"(smem_u32(dst)), "l"(map), "r"(bar_cluster_addr), "r"(x), "r"(y), "r"(z)
        : "memory");
}

struct FpTile { int m0, n0; };
__device__ __forceinline__ FpTile fp_tile(const F8PairParams &P, int tile)
{
    int g, r, tile_m, tile_n;
    P.d_group.divmod(tile, g, r);                        // by kFpGroupM * tiles_n
    const int rows_here = min(kFpGroupM, P.tiles_m - g * kFpGroupM);
    if (rows_here == kFpGroupM) { tile_n = r / kFpGroupM; tile_m = g * kFpGroupM + r % kFpGroupM; }
    else                        { tile_n = r / rows_here; tile_m = g * kFpGroupM + r % rows_here; }
    return {tile_m * 256, tile_n * P.bn};
}

struct FpMmaArgs {
    uint64_t *full_bar, *empty_bar, *acc_full, *acc_free;
    uint32_t ring, stage_bytes, a_bytes, b_bytes, tmem, a_desc_lo, b_desc_lo, idesc, buf1, set_col, set_cols, sets, stages;
    int k_blocks, tile0, tiles_total, tile_step, overlap;
};

// The issuing warp's loop; false when a wait ran out.  AK, BK: start-address steps (16-byte units) of 32 reduction bytes in the operands'
// layouts, RB: bytes of a row of an M/N-major B tile; BT: pieces of scales of B.
template <uint32_t AK, uint32_t BK, uint32_t RB, int BT>
__device__ __forceinline__ bool fp_mma_loop(const FpMmaArgs &A)
{
    constexpr uint32_t a_hi = (1024u >> 4) | (1u << 14) | (2u << 29);
    constexpr uint32_t b_hi = ((8u * RB) >> 4) | (1u << 14) | ((RB == 128 ? 2u : 4u) << 29);
    uint32_t s = 0, ph = 0, buf = 0, fph = 1, set = 0, at = A.ring, in_group = 0, group = 0;
    bool ready = false;                              // this lane has seen the next stage filled
    for (int tile = A.tile0; tile < A.tiles_total; tile += A.tile_step) {
        if (!mbar_wait_uniform(&A.acc_free[A.overlap ? 0u : buf], fph)) return false;
        if (A.overlap || buf == 1u) fph ^= 1u;
        tc_fence_after();
        const uint32_t d_tmem = A.tmem + buf * A.buf1;
        uint32_t t_sa = 0;
        for (int kb = 0; kb < A.k_blocks; ++kb) {
            if (!__all_sync(0xffffffffu, ready) && !mbar_wait_uniform(&A.full_bar[s], ph)) return false;
            tc_fence_after();
            const uint32_t here = at;
            at += A.stage_bytes;
            if (++s == A.stages) { s = 0; ph ^= 1u; at = A.ring; }
            ready = mbar_test(&A.full_bar[s], ph);
            if ((kb & 3) == 0) {
                set = set + 1 == A.sets ? 0u : set + 1;
                t_sa = A.tmem + A.set_col + set * A.set_cols;
                const uint32_t scales = here + A.a_bytes + A.b_bytes;
                if (elect_one()) {
                    copy_piece_pair(t_sa, piece_desc(scales));
#pragma unroll
                    for (int k = 0; k < BT; ++k) copy_piece_pair(t_sa + 4u + 4u * k, piece_desc(scales + kF8Piece * (1 + k)));
                }
            }
            const uint32_t id = (uint32_t)(kb & 3), idesc = A.idesc | (id << 4) | (id << 29);
            const uint32_t a_lo = ((here >> 4) & 0x3FFFu) | A.a_desc_lo, b_lo = (((here + A.a_bytes) >> 4) & 0x3FFFu) | A.b_desc_lo;
            if (elect_one()) {
#pragma unroll
                for (uint32_t kk = 0; kk < 4; ++kk)
                    mma_f8_pair(d_tmem, ((uint64_t)a_hi << 32) | (uint64_t)(a_lo + kk * AK), ((uint64_t)b_hi << 32) | (uint64_t)(b_lo + kk * BK),
                                idesc, t_sa, t_sa + 4u, kk == 0 && kb == 0 ? 0u : 1u);
            }
            if (++in_group == kFpRelease) {
                if (elect_one()) mma_commit_pair(&A.empty_bar[group]);
                in_group = 0;
                if (++group * kFpRelease == A.stages) group = 0;
            }
        }
        if (elect_one()) mma_commit_pair(&A.acc_full[buf]);
        buf ^= 1u;
    }
    return true;
}

// Accumulators of this lane's row as they are stored, 64 bytes of a swizzled slab row: 16 of fp32 or 32 of the halves.
__device__ __forceinline__ uint4 *fp_slab(uint8_t *slab, int lane, int piece) { return reinterpret_cast<uint4 *>(slab + lane * 64 + ((piece ^ ((lane >> 1) & 3)) << 4)); }
template <typename T> __device__ __forceinline__ void fp_slab_halves(uint8_t *slab, int lane, const uint32_t (&r)[32])
{
#pragma unroll
    for (int j = 0; j < 32; j += 8) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(r[j + e]);
        *fp_slab(slab, lane, j >> 3) = pack8<T>(v).w[0];
    }
}
template <typename T> __device__ __forceinline__ void fp_put(void *out, int64_t at, float v) { static_cast<T *>(out)[at] = real_to<T>(v); }

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kFpThreads, 1) f8_pair_kernel(const __grid_constant__ F8PairParams P)
{
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t full_bar[kFpMaxStages], empty_bar[kFpMaxStages / kFpRelease], acc_full[2], acc_free[2];
    __shared__ uint32_t tmem_slot;

    const uint32_t raw_addr = smem_u32(smem_raw);
    uint8_t *smem = smem_raw + ((1024u - (raw_addr & 1023u)) & 1023u);
    uint8_t *staging = smem + (size_t)P.stages * P.stage_bytes;              // 1024-aligned, as the stages are
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();                                 // 0: leader of the pair
    const int pair = blockIdx.x >> 1;

    if (threadIdx.x == 0) {
        // "full": the leader's arrive + the bytes of both CTAs; "empty" (of a release group) and "acc_full": one multicast commit each;
        // "acc_free" (the leader's is the one waited on): eight warps of each CTA
        for (int s = 0; s < P.stages; ++s) mbar_init(&full_bar[s], 1);
        for (int g = 0; g < P.stages / (int)kFpRelease; ++g) mbar_init(&empty_bar[g], 1);
        for (int b = 0; b < 2; ++b) { mbar_init(&acc_full[b], 1); mbar_init(&acc_free[b], 2 * kFpEpiWarps); }
        mbar_fence_init();
        tma_prefetch_desc(&P.mapA); tma_prefetch_desc(&P.mapB); tma_prefetch_desc(&P.mapSA); tma_prefetch_desc(&P.mapSB);
        if (P.tma_out) tma_prefetch_desc(&P.mapC);
    }
    if (warp == 1) { tmem_alloc_pair(&tmem_slot, 512); tmem_relinquish_pair(); }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();                  // both CTAs' barriers are initialised before either signals the other
    tc_fence_after();
    const uint32_t tmem_base = tmem_slot;
    bool timed_out = false;
    pdl_wait();
    // (cleared here and not by a launch of its own: a wait gives up a second after it began, long after a grid's first block has started)
    if (blockIdx.x == 0 && threadIdx.x == 0) *P.status = 0;

    if (warp == 0) {
        // (the whole warp in step, an elected lane issues: addresses and coordinates then stay in uniform registers, where the copies
        // want them; by one lane of a divergent warp a block's two copies took 500 cycles, as long as its MMAs)
        uint32_t s = 0, ph = 1, in_group = 0, group = 0;
        const uint32_t operand_bytes = 2u * (P.a.tile_bytes + P.b.tile_bytes), scale_bytes = 2u * (uint32_t)kF8Piece * (1u + (uint32_t)(P.bn >> 7));
        const uint32_t full0 = map_to_cta(&full_bar[0], 0);
        const bool a_k = P.a.major == 0, b_k = P.b.major == 0;
        for (int tile = pair; tile < P.tiles_total && !timed_out; tile += P.pairs) {
            const FpTile o = fp_tile(P, tile);
            const int m_mine = o.m0 + 128 * (int)rank, n_mine = o.n0 + (P.bn >> 1) * (int)rank;
            for (int kb = 0; kb < P.k_blocks; ++kb) {
                if (in_group == 0 && !mbar_wait_uniform(&empty_bar[group], ph)) { timed_out = true; break; }
                if (++in_group == kFpRelease) { in_group = 0; ++group; }
                uint8_t *sa = smem + (size_t)s * P.stage_bytes, *sb = sa + P.a.tile_bytes, *scales = sb + P.b.tile_bytes;
                const uint32_t bar = full0 + 8u * s;
                const bool with_scales = (kb & 3) == 0;
                const int k0 = kb * 128;
                if (elect_one()) {
                    if (rank == 0) mbar_expect_tx(&full_bar[s], operand_bytes + (with_scales ? scale_bytes : 0u));
                    tma_load_2d_pair(sa, &P.mapA, bar, a_k ? k0 : m_mine, a_k ? m_mine : k0);
                    tma_load_2d_pair(sb, &P.mapB, bar, b_k ? k0 : n_mine, b_k ? n_mine : k0);
                    if (with_scales) {
                        tma_load_3d_pair(scales, &P.mapSA, bar, 0, kb >> 2, m_mine >> 7);
                        tma_load_3d_pair(scales + kF8Piece, &P.mapSB, bar, 0, kb >> 2, o.n0 >> 7);
                    }
                }
                __syncwarp();
                if (++s == (uint32_t)P.stages) { s = 0; ph ^= 1u; group = 0; }
            }
        }
    } else if (warp == 1) {
        if (rank == 0) {
            FpMmaArgs A;
            A.full_bar = full_bar; A.empty_bar = empty_bar; A.acc_full = acc_full; A.acc_free = acc_free; A.overlap = P.overlap;
            A.ring = smem_u32(smem); A.stage_bytes = P.stage_bytes; A.a_bytes = P.a.tile_bytes; A.b_bytes = P.b.tile_bytes; A.tmem = tmem_base;
            A.a_desc_lo = P.a.desc_lo; A.b_desc_lo = P.b.desc_lo; A.idesc = P.idesc; A.buf1 = P.buf1; A.set_col = P.set_col;
            A.set_cols = P.set_cols; A.sets = P.sets; A.stages = (uint32_t)P.stages;
            A.k_blocks = P.k_blocks; A.tile0 = pair; A.tiles_total = P.tiles_total; A.tile_step = P.pairs;
            bool ok;
            if (P.bn == 256) {
                if (P.a.major == 0) ok = P.b.major == 0 ? fp_mma_loop<2, 2, 128, 2>(A) : fp_mma_loop<2, 256, 128, 2>(A);
                else                ok = P.b.major == 0 ? fp_mma_loop<256, 2, 128, 2>(A) : fp_mma_loop<256, 256, 128, 2>(A);
            } else {
                if (P.a.major == 0) ok = P.b.major == 0 ? fp_mma_loop<2, 2, 128, 1>(A) : fp_mma_loop<2, 128, 64, 1>(A);
                else                ok = P.b.major == 0 ? fp_mma_loop<256, 2, 128, 1>(A) : fp_mma_loop<256, 128, 64, 1>(A);
            }
            timed_out = !ok;
        }
    } else {
        // the two groups of four warps take half the columns each
        const int ew = warp - 2, quad = warp & 3, half = ew >> 2;
        uint8_t *slab = staging + (size_t)ew * kFpSlab;
        const uint32_t leader_free = map_to_cta(&acc_free[0], 0);
        const int per_half = P.bn >> 6;                                       // chunks of 32 columns
        uint32_t buf = 0, fph = 0;
        for (int tile = pair; tile < P.tiles_total; tile += P.pairs) {
            const FpTile o = fp_tile(P, tile);
            const int64_t m_slab = (int64_t)o.m0 + 128 * (int)rank + 32 * quad;
            // This warp's arrival, one a tile and behind the wait for the tile's MMAs, so that it counts for no other tile.  Shared columns:
            // the next tile's MMAs write the accumulator that this warp has drained before, and of this one the shared columns (the last of
            // the first accumulator, the first of the second), two chunks of one half's warps.  Else the accumulator is free once drained.
            const bool shares = buf == 0 ? half == 1 : half == 0;
            const int free_at = !P.overlap ? per_half - 1 : shares ? 1 : -1;
            const uint32_t free_bar = leader_free + (P.overlap ? 0u : 8u * buf);
            if (!timed_out && !mbar_wait_warp(&acc_full[buf], fph)) timed_out = true;
            if (timed_out || free_at < 0) { tc_fence_before(); __syncwarp(); if (lane == 0) mbar_arrive_cluster(free_bar); }
            if (!timed_out) {
                tc_fence_after();
                const uint32_t t_addr = tmem_base + ((uint32_t)(quad * 32) << 16) + buf * P.buf1;
                for (int i = 0; i < per_half; ++i) {
                    const int c0 = 32 * (half * per_half + (P.overlap && buf == 0 ? per_half - 1 - i : i));
                    uint32_t r[32];
                    tmem_ld_32x32(t_addr + (uint32_t)c0, r);
                    tmem_ld_wait();
                    if (i == free_at) { tc_fence_before(); __syncwarp(); if (lane == 0) mbar_arrive_cluster(free_bar); }
                    if (o.n0 + c0 >= P.N || m_slab >= P.M) continue;
                    if (P.tma_out && P.dtype == QBP_F32) {
#pragma unroll
                        for (int h = 0; h < 32; h += 16) {
                            if (lane == 0) tma_store_wait_read();
                            __syncwarp();
#pragma unroll
                            for (int j = 0; j < 16; j += 4) *fp_slab(slab, lane, j >> 2) = make_uint4(r[h + j], r[h + j + 1], r[h + j + 2], r[h + j + 3]);
                            fence_proxy_async();
                            __syncwarp();
                            if (lane == 0 && o.n0 + c0 + h < P.N) { tma_store_2d(&P.mapC, slab, o.n0 + c0 + h, (int)m_slab); tma_store_commit(); }
                        }
                    } else if (P.tma_out) {
                        if (lane == 0) tma_store_wait_read();
                        __syncwarp();
                        if (P.dtype == QBP_BF16) fp_slab_halves<__nv_bfloat16>(slab, lane, r);
                        else                     fp_slab_halves<__half>(slab, lane, r);
                        fence_proxy_async();
                        __syncwarp();
                        if (lane == 0) { tma_store_2d(&P.mapC, slab, o.n0 + c0, (int)m_slab); tma_store_commit(); }
                    } else {
                        // rows that no TMA store can start on: transposed through the slab sixteen columns at a time, two rows of 16 at once
                        uint32_t *words = reinterpret_cast<uint32_t *>(slab);
                        const int rows = (int)min((int64_t)32, P.M - m_slab);
#pragma unroll
                        for (int h = 0; h < 32; h += 16) {
#pragma unroll
                            for (int j = 0; j < 16; ++j) words[lane * 16 + (j ^ (lane >> 1 & 15))] = r[h + j];
                            __syncwarp();
                            const int64_t n = (int64_t)o.n0 + c0 + h + (lane & 15);
                            for (int k = lane >> 4; k < rows; k += 2) {
                                const float v = __uint_as_float(words[k * 16 + ((lane & 15) ^ (k >> 1 & 15))]);
                                const int64_t at = (m_slab + k) * P.N + n;
                                if (n < P.N) {
                                    if (P.dtype == QBP_F32) fp_put<float>(P.out, at, v);
                                    else if (P.dtype == QBP_BF16) fp_put<__nv_bfloat16>(P.out, at, v);
                                    else fp_put<__half>(P.out, at, v);
                                }
                            }
                            __syncwarp();
                        }
                    }
                }
            }
            buf ^= 1u;
            if (buf == 0) fph ^= 1u;
        }
        if (lane == 0) tma_store_wait_all();
        __syncwarp();
    }

    if (timed_out) { raise_timeout(P.status); __nanosleep(1000000); }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();                  // neither CTA retires while the other may still read its memory or signal it
    if (warp == 1) { __syncwarp(); tmem_dealloc_pair(tmem_base, 512); }
}

int launch_f8_pair(const F8Product &p, cudaStream_t st)
{
    F8PairParams P{};
    int rc;
    const auto tiles_of = [&](int64_t n) { return ((p.M + 255) / 256) * ((p.N + n - 1) / n); };
    const int pairs = sm_count() / 2;
    // tiles of 128 columns where they fit the pairs once: their epilogues and first stages are shorter (256 x 2048 x 8192 30.7 us, of 256
    // columns 34.8); in a second round they are slower (2048 x 2048 x 8192 53.2 and 38.9)
    P.bn = tiles_of(128) > pairs ? 256 : 128;
    const uint32_t half = (uint32_t)P.bn / 2;
    if (!p.transA) { P.a = layout_kmajor(128, 128);         rc = make_map_2d(&P.mapA, p.A, p.M, p.K, 128, 128); }
    else           { P.a = layout_mnmajor(128, 128, 1, 0);  rc = make_map_2d(&P.mapA, p.A, p.K, p.M, 128, 128); }
    if (rc) return rc;
    if (p.transB)  { P.b = layout_kmajor(half, 128);        rc = make_map_2d(&P.mapB, p.B, p.N, p.K, half, 128); }
    else           { P.b = layout_mnmajor(128, half, 1, 0); rc = make_map_2d(&P.mapB, p.B, p.K, p.N, 128, half); }
    if (rc) return rc;
    if ((rc = make_map_scales(&P.mapSA, p.sA, p.M, p.K, 1)) || (rc = make_map_scales(&P.mapSB, p.sB, p.N, p.K, (uint32_t)P.bn / 128))) return rc;
    P.tma_out = aligned16(p.out) && p.N * (int64_t)dtype_size(p.dtype) % 16 == 0 ? 1 : 0;
    if (P.tma_out && (rc = make_map_out_rows64(&P.mapC, p.out, p.M, p.N, p.dtype))) return rc;
    P.idesc = make_idesc_f8(p.formatA, p.formatB, P.a.major, P.b.major, 256, (uint32_t)P.bn);
    P.k_blocks = (int)f8_blocks(p.K);
    P.overlap = P.bn == 256 ? 1 : 0;
    P.buf1 = P.bn == 256 ? 192u : 128u;
    P.set_col = P.bn == 256 ? 448u : 256u;
    P.set_cols = P.bn == 256 ? 12u : 8u;
    P.sets = P.bn == 256 ? 5u : 8u;
    P.tiles_m = (int)((p.M + 255) / 256); P.tiles_n = (int)((p.N + P.bn - 1) / P.bn);
    const int64_t total = (int64_t)P.tiles_m * P.tiles_n;
    if (total > (1 << 30)) return fail(QBP_ERR_UNSUPPORTED_SHAPE, "gemm_f8: %lld output tiles", (long long)total);
    P.tiles_total = (int)total;
    P.pairs = std::min(P.tiles_total, pairs);
    P.d_group = make_fastdiv(kFpGroupM * P.tiles_n);
    P.stage_bytes = (uint32_t)align_up(P.a.tile_bytes + P.b.tile_bytes + (uint32_t)kF8Piece * (1u + (uint32_t)P.bn / 128u), 1024);   // 34 or 25 KB
    P.stages = std::min<int>(kFpMaxStages, (int)((kFpSmem - 1024 - kFpEpiWarps * kFpSlab) / P.stage_bytes));
    P.stages -= P.stages % (int)kFpRelease;                          // 6 or 8
    static_assert(kFpMaxStages + kFpRelease <= 17, "a set of scales is written again while MMAs may read it");
    P.M = p.M; P.N = p.N; P.out = p.out; P.dtype = p.dtype; P.status = p.status;
    const size_t smem = 1024 + (size_t)P.stages * P.stage_bytes + kFpEpiWarps * kFpSlab;
    static PerDeviceOnce configured;
    QBP_SMEM_OPT_IN(configured, f8_pair_kernel, kFpSmem);
    QBP_TRACE_BEGIN(st);
    launch(f8_pair_kernel, 2 * P.pairs, kFpThreads, smem, st, P);
    QBP_LAUNCH_OK("f8_pair_kernel");
    return QBP_OK;
}

}  // namespace qbp
