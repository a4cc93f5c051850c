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

// What a weight is held in: a probability, 2^8 at most (kRowsRebase), times its value's
// scale, 2^120 at most, would be infinite as 2^128; the rows' last factor takes the half
// back.  A weight of 2^-25 of the row's largest is still normal under a scale of 2^-100.
constexpr float kWeightUnit = 0.5f;

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

// Sum and maximum over the lanes that hold a row of 16: l, l + 16, l + 32, l + 48.
__device__ __forceinline__ float rows8_quad_sum(float x)
{
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false,
                                              false);
    return rows_pair_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}
__device__ __forceinline__ float rows8_quad_max(float x)
{
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false,
                                              false);
    return rows_pair_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}

// Four elements of key j of a tile, from d on (a multiple of four), as numbers.
template <int D>
__device__ __forceinline__ void rows8_values(const unsigned char *tile, int j, int d,
                                             float (&v)[4])
{
    const uint32_t w = *reinterpret_cast<const uint32_t *>(
        tile + j * D + (((d >> 4) ^ rows8_swz<D>(j)) << 4) + (d & 15));
    uint32_t x[2];
    q8_to_bf16(w, 1.f, x[0], x[1]);
#pragma unroll
    for (int e = 0; e < 4; ++e)
        v[e] = __uint_as_float(e & 1 ? x[e / 2] & 0xffff0000u : x[e / 2] << 16);
}

// Whether a tile of BYTES holds a NaN element (there are no infinite ones).
template <int BYTES>
__device__ __forceinline__ bool rows8_odd_elements(const unsigned char *vt, int lane)
{
    uint32_t carry = 0;
#pragma unroll
    for (int i = 0; i < BYTES / 1024; ++i) {
        const u32x4 w = *reinterpret_cast<const u32x4 *>(vt + i * 1024 + lane * 16);
#pragma unroll
        for (int e = 0; e < 4; ++e)  // 0x7f carries into the sign bit
            carry |= (w[e] & 0x7f7f7f7fu) + 0x01010101u;
    }
    return __builtin_amdgcn_ballot_w64((carry & 0x80808080u) != 0) != 0;
}

// One wave's 32 rows against 8-bit tiles of NKB 32-key blocks.  K: a lane's fragment
// is eight elements of one key, so that the conversion applies the key's scale; the
// two of a 16-byte read go to two products, and Q is held in the same order of d.  V:
// a fragment is eight keys of one d, whose scales go to their probabilities instead.
template <int D, int NKB, int SCORE>
struct RowBlock8 : RowBlock<D, NKB, SCORE> {
    using Base = RowBlock<D, NKB, SCORE>;
    using Base::col;
    using Base::half;
    using Base::oacc;
    using Base::qf;
    static constexpr int READS = D / 32;  // 16-byte reads of a key
    static constexpr int D_BLOCKS = D / 32;
    static constexpr int CHUNKS = D / 8;  // of four sums of this lane's row
    using Scores = f32x16[NKB];
    using Probs = bf16x8[NKB][2];

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

    // Where this lane's i-th fragment of Q lies in its row, in 16-byte chunks.
    __device__ __forceinline__ int q_chunk(int i) const { return 4 * (i >> 1) + 2 * half + (i & 1); }
    static constexpr int Q_FRAGMENTS = D / 16;

    __device__ __forceinline__ bool first() const { return half == 0; }
    __device__ __forceinline__ float row_sum(float x) const { return rows_pair_sum(x); }
    __device__ __forceinline__ f32x4r chunk(int c) const
    {
        f32x4r x;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            x[e] = oacc[c / 4][4 * (c % 4) + e];
        return x;
    }
    __device__ __forceinline__ int chunk_d(int c) const { return 8 * c + 4 * half; }

    // Raw products; scales: the bytes of the tile's keys.
    __device__ __forceinline__ void products8(const unsigned char *kt, const unsigned char *scales,
                                              Scores &s) const
    {
        float f[NKB];
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb) {
            f[kb] = q8_scale_bits(scales[kb * 32 + rows_perm(col)]);
            s[kb] = f32x16{};
        }
#pragma unroll
        for (int t = 0; t < READS; ++t)
#pragma unroll
            for (int kb = 0; kb < NKB; ++kb) {
                const u32x4 w =
                    *reinterpret_cast<const u32x4 *>(kt + koff8[t] + kb * 32 * D);
                s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                    q8_fragment(w[0], w[1], f[kb]), qf[2 * t], s[kb], 0, 0, 0);
                s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                    q8_fragment(w[2], w[3], f[kb]), qf[2 * t + 1], s[kb], 0, 0, 0);
            }
    }

    // softmax() whose weights carry the values' scales (fp32 in kWeightUnit, one a key of
    // the tile).
    __device__ __forceinline__ void softmax8(const Scores &s, const ScoreArgs &a, float slope_log2,
                                             int dist0, Probs &p, bool fresh, const float *scales)
    {
        f32x4r w[NKB][4];  // of this lane's keys (rows_key_of_reg)
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                w[kb][i] = *reinterpret_cast<const f32x4r *>(scales + 32 * kb + 16 * (i >> 1) +
                                                             8 * half + 4 * (i & 1));
        this->softmax(s, a, slope_log2, dist0, p, fresh,
                      [&](int kb, int v, float x) TA_INLINE { return x * w[kb][v / 4][v % 4]; });
    }

    // O^T += V^T P^T, P with the values' scales.
    __device__ __forceinline__ void accumulate8(const unsigned char *vt, const Probs &pf)
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

    // accumulate8() key by key, each only to the rows that keep it.
    __device__ __forceinline__ void accumulate8_by_key(const unsigned char *vt, const Scores &x,
                                                       const Probs &pf)
    {
#pragma unroll 1
        for (int j = 0; j < NKB * 32; ++j) {
            float p;
            const bool keeps = this->weight_of_key(j, x, pf, p);
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                float v[4];
                rows8_values<D>(vt, j, chunk_d(c), v);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    oacc[c / 4][4 * (c % 4) + e] += keeps ? p * v[e] : 0.f;
            }
        }
    }
};

// One wave's 16 rows against 8-bit tiles, for the calls whose requests have no more
// (single tokens): half the matrix and softmax work of 32 columns that mostly stand
// empty.  S^T = K Q^T by MFMA 16x16x32, a 32-key block as two of 16 rows: row
// 4 u + i of part b is key 8 u + 4 (b ^ (u & 1)) + i, which leaves the scores of keys
// 8 u .. 8 u + 7 in the lanes of quarter u, as the other product wants them, and lets
// eight rows that follow one another read K in different banks.
template <int D, int NKB, int SCORE>
struct RowBlock8x16 {
    static constexpr int READS = D / 64;  // 16-byte reads of a key, four quarters each
    static constexpr int D_BLOCKS = D / 16;
    static constexpr int CHUNKS = D_BLOCKS;
    static constexpr int Q_FRAGMENTS = D / 32;
    using Scores = f32x4r[NKB][2];
    using Probs = bf16x8[NKB];

    bf16x8 qf[Q_FRAGMENTS];
    f32x4r oacc[D_BLOCKS];
    float m_ref;  // as in RowBlock
    float l_run;
    uint32_t koff[2][READS];
    uint32_t voff[D_BLOCKS];
    int key[2];   // this lane's first key of part b
    int krow[2];  // the key whose K elements it reads for part b
    int quarter, col;

    __device__ __forceinline__ void init(int lane)
    {
        quarter = lane >> 4;
        col = lane & 15;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            key[b] = 8 * quarter + 4 * (b ^ (quarter & 1));
            const int u = col >> 2;
            krow[b] = 8 * u + 4 * (b ^ (u & 1)) + (col & 3);
#pragma unroll
            for (int t = 0; t < READS; ++t)
                koff[b][t] = (uint32_t)(krow[b] * D +
                                        (((4 * t + quarter) ^ rows8_swz<D>(krow[b])) << 4));
        }
        // transposed reads as in RowBlock8, the rows of an odd quarter in the order
        // of its scores: 4 .. 7, 0 .. 3
        const int vrow = 8 * quarter + ((col >> 1) ^ (4 * (quarter & 1)));
#pragma unroll
        for (int b = 0; b < D_BLOCKS; ++b)
            voff[b] = (uint32_t)(vrow * D + ((b ^ rows8_swz<D>(vrow)) << 4) + 8 * (col & 1));
    }

    __device__ __forceinline__ int q_chunk(int i) const
    {
        return 8 * (i >> 1) + 2 * quarter + (i & 1);
    }
    __device__ __forceinline__ bool first() const { return quarter == 0; }
    __device__ __forceinline__ float row_sum(float x) const { return rows8_quad_sum(x); }
    __device__ __forceinline__ f32x4r chunk(int c) const { return oacc[c]; }
    __device__ __forceinline__ int chunk_d(int c) const { return 16 * c + 4 * quarter; }

    __device__ __forceinline__ void reset()
    {
#pragma unroll
        for (int b = 0; b < D_BLOCKS; ++b)
            oacc[b] = f32x4r{};
        m_ref = -INFINITY;
        l_run = 0.f;
    }

    __device__ __forceinline__ void products8(const unsigned char *kt, const unsigned char *scales,
                                              Scores &s) const
    {
        float f[NKB][2];
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                f[kb][b] = q8_scale_bits(scales[kb * 32 + krow[b]]);
                s[kb][b] = f32x4r{};
            }
#pragma unroll
        for (int t = 0; t < READS; ++t)
#pragma unroll
            for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const u32x4 w =
                        *reinterpret_cast<const u32x4 *>(kt + koff[b][t] + kb * 32 * D);
                    s[kb][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                        q8_fragment(w[0], w[1], f[kb][b]), qf[2 * t], s[kb][b], 0, 0, 0);
                    s[kb][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                        q8_fragment(w[2], w[3], f[kb][b]), qf[2 * t + 1], s[kb][b], 0, 0, 0);
                }
    }

    // As RowBlock::modify, mask_above and softmax.
    __device__ __forceinline__ void modify(Scores &s, const ScoreArgs &a) const
    {
        if constexpr ((SCORE & kScoreCap) != 0) {
#pragma unroll
            for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        s[kb][b][i] = __builtin_amdgcn_rcpf(
                            -1.f - __builtin_amdgcn_exp2f(s[kb][b][i] * a.cap_in));
        }
    }
    __device__ __forceinline__ void mask_above(Scores &s, int lim) const
    {
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    s[kb][b][i] = kb * 32 + key[b] + i <= lim ? s[kb][b][i] : -INFINITY;
    }
    __device__ __forceinline__ void softmax8(const Scores &s, const ScoreArgs &a, float slope_log2,
                                             int dist0, Probs &p, bool fresh, const float *scales)
    {
        f32x4r w[NKB][2];
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
            for (int b = 0; b < 2; ++b)
                w[kb][b] = *reinterpret_cast<const f32x4r *>(scales + 32 * kb + key[b]);
        const float f = RowBlock<D, NKB, SCORE>::factor(a);
        const float offset = (SCORE & kScoreCap) != 0 ? a.cap_out : 0.f;
        float base[2] = {offset, offset};
        if constexpr ((SCORE & kScoreSlope) != 0)
#pragma unroll
            for (int b = 0; b < 2; ++b)
                base[b] = __builtin_fmaf(slope_log2, (float)(dist0 + key[b]), offset);
        auto score = [&](int kb, int b, int i, float m) TA_INLINE -> float {
            float x = base[b] - m;
            if constexpr ((SCORE & kScoreSlope) != 0)
                x = __builtin_fmaf(slope_log2, (float)(kb * 32 + i), x);
            return __builtin_fmaf(s[kb][b][i], f, x);
        };
        auto exps = [&](float m) TA_INLINE -> float {
            float sum[2] = {0.f, 0.f};
#pragma unroll
            for (int kb = 0; kb < NKB; ++kb) {
                u32x4 packed;
#pragma unroll
                for (int v = 0; v < 8; v += 2) {
                    typedef float f32x2r __attribute__((ext_vector_type(2)));
                    f32x2r t;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int b = v / 4, i = v % 4 + e;
                        t[e] = __builtin_amdgcn_exp2f(score(kb, b, i, m));
                        sum[e] += t[e];
                        t[e] *= w[kb][b][i];
                    }
                    packed[v / 2] =
                        __builtin_bit_cast(uint32_t, __builtin_convertvector(t, bf16x2q));
                }
                p[kb] = __builtin_bit_cast(bf16x8, packed);
            }
            return sum[0] + sum[1];
        };
        float sum = INFINITY;
        if (!fresh)
            sum = exps(m_ref);
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(sum <= kRowsRebase)) != 0, 0)) {
            float mx = -INFINITY;
#pragma unroll
            for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        mx = fmaxf(mx, score(kb, b, i, 0.f));
            mx = rows8_quad_max(mx);
            // only the rows that need it
            const bool mine = rows8_quad_max(sum <= kRowsRebase ? 0.f : 1.f) != 0.f;
            const float m_new = mine ? fmaxf(m_ref, mx) : m_ref;
            const float m_use = m_new == -INFINITY ? 0.f : m_new;
            const float alpha = __builtin_amdgcn_exp2f(m_ref - m_use);
            l_run *= alpha;
#pragma unroll
            for (int b = 0; b < D_BLOCKS; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    oacc[b][i] *= alpha;
            m_ref = m_new;
            sum = exps(m_use);
        }
        l_run += sum;
    }

    __device__ __forceinline__ void accumulate8(const unsigned char *vt, const Probs &p)
    {
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
            for (int b = 0; b < D_BLOCKS; ++b) {
                const i32x2r w = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                    (lds_i32x2r *)(vt + voff[b] + kb * 32 * D));
                oacc[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                    q8_fragment((uint32_t)w[0], (uint32_t)w[1], 1.f), p[kb], oacc[b], 0, 0, 0);
            }
    }

    // accumulate8() key by key, each only to the rows that keep it.
    __device__ __forceinline__ void accumulate8_by_key(const unsigned char *vt, const Scores &x,
                                                       const Probs &p)
    {
        typedef uint16_t u16x8r __attribute__((ext_vector_type(8)));
#pragma unroll 1
        for (int j = 0; j < NKB * 32; ++j) {
            float mine = 0.f, kept = 0.f;
#pragma unroll
            for (int kb = 0; kb < NKB; ++kb) {
                const u16x8r pb = __builtin_bit_cast(u16x8r, p[kb]);
#pragma unroll
                for (int v = 0; v < 8; ++v) {
                    const bool on = kb * 32 + key[v / 4] + v % 4 == j;
                    mine = on ? __uint_as_float((uint32_t)pb[v] << 16) : mine;
                    kept = on && x[kb][v / 4][v % 4] != -INFINITY ? 1.f : kept;
                }
            }
            const float w = rows8_quad_sum(mine);
            const bool keeps = rows8_quad_sum(kept) != 0.f;
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                float v[4];
                rows8_values<D>(vt, j, chunk_d(c), v);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    oacc[c][e] += keeps ? w * v[e] : 0.f;
            }
        }
    }
};

}  // namespace triattn
