// Row blocks over K/V tiles that are held in 8 bits: the form of the cache, its
// conversions, and the row-block core's products on 8-bit tiles in LDS.  Not part
// of the public interface.
//
// Mathematics.  A row (one kv head of one token) is held as e4m3 elements c and a
// scale 2^e, one byte e + 127: its values are c 2^e.  A power of two, because it
// then rounds nothing: the conversion to bf16 applies it (four significant bits
// always fit bf16's eight), and a probability times it is exact.  In a format of
// floating-point elements a scale's mantissa would gain less than one power of two
// of range, and no precision.
#pragma once

#include "triattn_rows.h"

namespace triattn {

typedef int i32x2r __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) i32x2r lds_i32x2r;
typedef __bf16 bf16x2q __attribute__((ext_vector_type(2)));

// Scales 2^e that are written: e in kLeastExp .. kMostExp.
constexpr int kLeastExp = -100, kMostExp = 120;

// The fp32 number whose exponent field is a scale's byte, as the conversions take
// a scale (they read 0 as 2^-127 and 255 as NaN).
__device__ __forceinline__ float q8_scale_bits(uint32_t byte)
{
    return __uint_as_float(byte << 23);
}

// The scale itself: 2^(byte - 127), NaN for 255.
__device__ __forceinline__ float q8_scale(uint32_t byte)
{
    return __uint_as_float((byte << 23) | (byte - 1 >= 254 ? 0x00400000u : 0u));
}

// Four elements times a scale, in bf16: exact, but for values past bf16's range.
__device__ __forceinline__ void q8_to_bf16(uint32_t four, float scale_bits, uint32_t &lo,
                                           uint32_t &hi)
{
    lo = __builtin_bit_cast(uint32_t,
                            __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(four, scale_bits, false));
    hi = __builtin_bit_cast(uint32_t,
                            __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(four, scale_bits, true));
}

__device__ __forceinline__ bf16x8 q8_fragment(uint32_t w0, uint32_t w1, float scale_bits)
{
    u32x4 x;
    uint32_t a, b, c, d;
    q8_to_bf16(w0, scale_bits, a, b);
    q8_to_bf16(w1, scale_bits, c, d);
    x[0] = a;
    x[1] = b;
    x[2] = c;
    x[3] = d;
    return __builtin_bit_cast(bf16x8, x);
}

// 16-byte chunk swizzle of 8-bit LDS tiles ([key][d] rows of D bytes): eight keys
// that follow one another then lie in different banks, for K's 16-byte reads and
// V's transposed ones alike.
template <int D>
__device__ __forceinline__ int rows8_swz(int r)
{
    return D == 128 ? (r & 7) : ((r >> 1) & 3);
}

// One wave's 32 rows against 8-bit tiles.  K: a lane's fragment is eight elements
// of one key, so that the conversion applies the key's scale; the two of a 16-byte
// read go to two products, and Q is loaded in the same order of d.  V: a fragment
// is eight keys of one d, whose scales go to their probabilities instead.
template <int D, int NKB, int SCORE>
struct RowBlock8 : RowBlock<D, NKB, SCORE> {
    using Base = RowBlock<D, NKB, SCORE>;
    using Base::col;
    using Base::half;
    using Base::oacc;
    using Base::qf;
    static constexpr int READS = D / 32;  // 16-byte reads of a key
    static constexpr int D_BLOCKS = D / 32;

    uint32_t koff8[READS];
    uint32_t voff8[D_BLOCKS];

    __device__ __forceinline__ void init(int lane)
    {
        half = lane >> 5;
        col = lane & 31;
        const int krow = rows_perm(col);
#pragma unroll
        for (int t = 0; t < READS; ++t)
            koff8[t] = (uint32_t)(krow * D + (((2 * t + half) ^ rows8_swz<D>(krow)) << 4));
        // transposed reads: in each group of 16 lanes, lane i addresses row
        // K0 + i / 2 at d = D0 + 8 (i % 2), and lane j receives rows K0 .. K0 + 7
        // at d = D0 + j
        const int vrow = 8 * half + ((lane & 15) >> 1);
#pragma unroll
        for (int b = 0; b < D_BLOCKS; ++b)
            voff8[b] = (uint32_t)(vrow * D +
                                  (((2 * b + ((lane >> 4) & 1)) ^ rows8_swz<D>(vrow)) << 4) +
                                  8 * (lane & 1));
    }

    __device__ __forceinline__ void load_q(const uint16_t *row)
    {
#pragma unroll
        for (int s = 0; s < D / 16; ++s)
            qf[s] = *reinterpret_cast<const bf16x8 *>(row + 32 * (s >> 1) + 16 * half +
                                                      8 * (s & 1));
    }

    // Raw products; scale_bits[kb]: of this lane's key, rows_perm(col), of block kb.
    __device__ __forceinline__ void products8(const unsigned char *kt,
                                              const float (&scale_bits)[NKB],
                                              f32x16 (&s)[NKB]) const
    {
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb)
            s[kb] = f32x16{};
#pragma unroll
        for (int t = 0; t < READS; ++t)
#pragma unroll
            for (int kb = 0; kb < NKB; ++kb) {
                const u32x4 w =
                    *reinterpret_cast<const u32x4 *>(kt + koff8[t] + kb * 32 * D);
                s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                    q8_fragment(w[0], w[1], scale_bits[kb]), qf[2 * t], s[kb], 0, 0, 0);
                s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                    q8_fragment(w[2], w[3], scale_bits[kb]), qf[2 * t + 1], s[kb], 0, 0, 0);
            }
    }

    // O^T += V^T P^T, P with the values' scales.
    __device__ __forceinline__ void accumulate8(const unsigned char *vt,
                                                const bf16x8 (&pf)[NKB][2])
    {
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
            for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
                for (int b = 0; b < D_BLOCKS; ++b) {
                    const i32x2r w = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                        (lds_i32x2r *)(vt + voff8[b] + (kb * 32 + s2 * 16) * D));
                    oacc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                        q8_fragment((uint32_t)w[0], (uint32_t)w[1], 1.f), pf[kb][s2], oacc[b], 0,
                        0, 0);
                }
    }

    // Whether a tile holds a NaN element (there are no infinite ones).
    __device__ __forceinline__ static bool odd_elements(const unsigned char *vt, int lane)
    {
        uint32_t carry = 0;
#pragma unroll
        for (int i = 0; i < NKB * 32 * D / 1024; ++i) {
            const u32x4 w = *reinterpret_cast<const u32x4 *>(vt + i * 1024 + lane * 16);
#pragma unroll
            for (int e = 0; e < 4; ++e)  // 0x7f carries into the sign bit
                carry |= (w[e] & 0x7f7f7f7fu) + 0x01010101u;
        }
        return __builtin_amdgcn_ballot_w64((carry & 0x80808080u) != 0) != 0;
    }

    // accumulate8() key by key, each only to the rows that keep it.
    __device__ __forceinline__ void accumulate8_by_key(const unsigned char *vt,
                                                       const f32x16 (&x)[NKB],
                                                       const bf16x8 (&pf)[NKB][2])
    {
#pragma unroll 1
        for (int j = 0; j < NKB * 32; ++j) {
            float p;
            const bool keeps = this->weight_of_key(j, x, pf, p);
            const unsigned char *row = vt + j * D;
#pragma unroll
            for (int b = 0; b < D_BLOCKS; ++b)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    // accumulators 4 c .. 4 c + 3: d = 32 b + 8 c + 4 half ..
                    const uint32_t w = *reinterpret_cast<const uint32_t *>(
                        row + (((2 * b + (c >> 1)) ^ rows8_swz<D>(j)) << 4) + 8 * (c & 1) +
                        4 * half);
                    uint32_t v[2];
                    q8_to_bf16(w, 1.f, v[0], v[1]);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        oacc[b][4 * c + e] +=
                            keeps ? p * __uint_as_float(e & 1 ? v[e / 2] & 0xffff0000u
                                                              : v[e / 2] << 16)
                                  : 0.f;
                }
        }
    }
};

}  // namespace triattn
