// 8-bit floating-point codes with a power-of-two scale for each block of 128: the format's constants, the scales' layout,
// and the tensor-core instructions that take them.
//
// Scales.  An operand of a product has an outer extent R (its rows or columns in the output) and a reduction extent K.  A
// scale belongs to one outer index and 128 consecutive reduction indices; it is stored as the byte e + 127 (255: not a
// number).  Bytes lie in pieces of 512 for 128 outer indices and 4 blocks, [ceil(R / 128)][ceil(K / 512)][512], the byte of
// outer index r and block b at (r % 32) * 16 + (r / 32 % 4) * 4 + b % 4 of its piece.  A piece is then, as it lies in memory,
// what one tcgen05.cp of 32 rows x 128 bits puts into four columns of tensor memory: lane r % 32, column r / 32, byte b % 4.
#pragma once

#include "qbp_mma.cuh"
#include "qbp_real.cuh"

namespace qbp {

constexpr int kF8Block = 128;
constexpr int kF8Piece = 512;                                    // bytes of scales for 128 outer indices x 4 blocks
inline int64_t f8_blocks(int64_t k) { return (k + 127) / 128; }
inline int64_t f8_groups(int64_t k) { return (k + 511) / 512; }

// Scales as 128 words x groups x tiles of 128 outer indices, read in boxes of `tiles` pieces (qbp_mma.cu).
int make_map_scales(CUtensorMap *map, const void *base, uint64_t outer, uint64_t K, uint32_t tiles);
// Output [rows x cols] of 4- or 2-byte elements stored in boxes of 32 rows of 64 bytes, swizzled alike (qbp_mma.cu).
int make_map_out_rows64(CUtensorMap *map, void *base, uint64_t rows, uint64_t cols, int dtype);

// Instruction descriptor of kind::mxf8f6f4: A / B type in bits 7..9 / 10..12 (0 = e4m3, 1 = e5m2), majors in 15 / 16, N >> 3 in
// 17..22, power-of-two scales in 23, M >> 4 in 24..28; the byte of a scale's word in 4..5 (B) and 29..30 (A).
inline uint32_t make_idesc_f8(int format_a, int format_b, uint32_t a_major, uint32_t b_major, uint32_t m, uint32_t n)
{
    return ((uint32_t)format_a << 7) | ((uint32_t)format_b << 10) | (a_major << 15) | (b_major << 16) | ((n >> 3) << 17) | (1u << 23) |
           ((m >> 4) << 24);
}

// One product, checked and split into what the kernels want (qbp_f8.cu): op(A) [M x K], op(B) [K x N].
struct F8Product {
    int transA, transB; int64_t M, N, K;
    int formatA, formatB;
    const uint8_t *A, *sA, *B, *sB;
    void *out; int dtype;
    int *status;
};
int launch_f8_pair(const F8Product &p, cudaStream_t st);

#ifdef __CUDACC__

template <typename T> struct IsBf16 { static constexpr bool value = false; };
template <> struct IsBf16<__nv_bfloat16> { static constexpr bool value = true; };

// Format constants: the largest value is 1.75 * 2^top.
template <int FORMAT> struct F8Format;
template <> struct F8Format<QBP_E4M3> { static constexpr int top = 8; };
template <> struct F8Format<QBP_E5M2> { static constexpr int top = 15; };

// Four values to codes, nearest with ties to even, saturating, the first in the lowest byte; a NaN to the format's NaN (0x7F).
template <int FORMAT> __device__ __forceinline__ uint32_t f8_codes4(float a, float b, float c, float d)
{
    uint32_t r;
    if (FORMAT == QBP_E4M3)
        asm("{\n\t.reg .b16 lo, hi;\n\tcvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n\tmov.b32 %0, {lo, hi};\n\t}" : "=r"(r) : "f"(a), "f"(b), "f"(c), "f"(d));
    else
        asm("{\n\t.reg .b16 lo, hi;\n\tcvt.rn.satfinite.e5m2x2.f32 lo, %2, %1;\n\tcvt.rn.satfinite.e5m2x2.f32 hi, %4, %3;\n\tmov.b32 %0, {lo, hi};\n\t}" : "=r"(r) : "f"(a), "f"(b), "f"(c), "f"(d));
    return r;
}
// Two products in one instruction.
__device__ __forceinline__ void mul2(float &a, float &b, float x, float y)
{
    asm("{\n\t.reg .b64 p, q;\n\tmov.b64 p, {%0, %1};\n\tmov.b64 q, {%2, %3};\n\tmul.rn.f32x2 p, p, q;\n\tmov.b64 {%0, %1}, p;\n\t}" : "+f"(a), "+f"(b) : "f"(x), "f"(y));
}
// Largest magnitude of three; NaN if one of them is.
__device__ __forceinline__ float amax3(float a, float b, float c)
{
    float d;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// The scale byte of a block from its largest magnitude: the smallest e >= -127 with amax <= 1.75 * 2^(top + e); 127 (a scale of
// one) for a block of zeros, 255 where a value is infinite or not a number.
template <int FORMAT> __device__ __forceinline__ uint32_t f8_scale_byte(float amax)
{
    const uint32_t bits = __float_as_uint(amax) & 0x7FFFFFFFu;
    if (bits >= 0x7F800000u) return 255u;
    if (bits == 0u) return 127u;
    const int e = (int)(bits >> 23) - 127 - F8Format<FORMAT>::top + ((bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return (uint32_t)(max(e, -127) + 127);
}
// 2^-e of a scale byte (e <= 120: a normal number, up to 2^127; NaN of 255)
__device__ __forceinline__ float f8_inverse(uint32_t byte) { return byte == 255u ? __uint_as_float(0x7FC00000u) : __uint_as_float((254u - byte) << 23); }
// Eight scaled values to eight codes.
template <int FORMAT> __device__ __forceinline__ uint2 f8_codes8(const float (&v)[8])
{
    return make_uint2(f8_codes4<FORMAT>(v[0], v[1], v[2], v[3]), f8_codes4<FORMAT>(v[4], v[5], v[6], v[7]));
}

// The larger of two magnitudes, of the halves two to a word as they are held.  A NaN is passed on.
template <typename T> struct HalfMax {
    static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b)
    {
        uint32_t r;
        if (sizeof(T) == 2 && IsBf16<T>::value) asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        else asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    static __device__ __forceinline__ float value(uint32_t w, int high)
    {
        const uint16_t h = (uint16_t)(high ? w >> 16 : w);
        T t;
        memcpy(&t, &h, 2);
        return real_of(t);
    }
};
// Whether the barrier's phase is complete, without waiting (try_wait may hold the thread for microseconds where it is not).
__device__ __forceinline__ bool mbar_test(uint64_t *bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
    return ok != 0;
}
// Descriptor of a piece of scales in shared memory (no swizzle, groups of 8 rows of 16 bytes 128 bytes apart).
__device__ __forceinline__ uint64_t piece_desc(uint32_t smem_addr)
{
    constexpr uint32_t hi = (128u >> 4) | (1u << 14);
    return ((uint64_t)hi << 32) | (uint64_t)((smem_addr >> 4) & 0x3FFFu);
}
// A piece of scales to four columns of tensor memory, the same in all four lane quarters.  In order with the MMAs that the
// same thread issues behind it; what read the columns before has to be complete.
__device__ __forceinline__ void copy_piece(uint32_t tmem, uint64_t desc)
{
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
__device__ __forceinline__ void copy_piece_pair(uint32_t tmem, uint64_t desc)
{
    asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
__device__ __forceinline__ void mma_f8(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t sa_tmem, uint32_t sb_tmem,
                                       uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%5], [%6], p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(sa_tmem), "r"(sb_tmem));
}
__device__ __forceinline__ void mma_f8_pair(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t sa_tmem, uint32_t sb_tmem,
                                            uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%5], [%6], p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(sa_tmem), "r"(sb_tmem));
}

#endif  // __CUDACC__
}  // namespace qbp
