// Row-block core of the paged and scored attention kernels of libtriattn.so:
// 32 query rows of one wave against K/V tiles in LDS, with an online softmax
// over modified scores.  Not part of the public interface.
//
// Mathematics.  For a row i and a key j,
//   x = softmax_scale <q_i, k_j>,  x <- cap tanh(x / cap) where a cap is set,
//   x <- x - slope (i - j) where slopes are set,
// and over the kept keys O = sum exp(x - m) v / sum exp(x - m) with a running
// reference m (one pass).  Scores are carried in the log2 domain, so that the
// exponentials are single exp2 instructions:
//   cap tanh(x / cap) = cap (1 - 2 / (1 + e^(2 x / cap))),
// one exp2, one reciprocal and three plain operations.  Its absolute error is at
// most 10 2^-24 of the cap, term by term (exponent 1.5, exp2 1, sum 2, reciprocal
// 2, the cap's factor 1.2, difference to the reference 2); 5.4 were measured.
//
// Layout, as in the forward tile kernel: S^T = K Q^T by bf16 MFMA 32x32x16
// (keys on the rows, queries on the columns), so that a lane holds scores of
// one query (column lane & 31) and softmax state is per lane.  The K rows are
// fed with bits 2 and 3 of the row index swapped, which makes the score
// registers directly the B operand of O^T += V^T P^T; V^T comes from
// transposed LDS reads.  Probabilities are rounded to bf16 for that product
// (half a step, 2^-8 relative, under bf16 inputs); row sums and the output
// accumulators stay fp32.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "triattn_device.h"

namespace triattn {

typedef float f32x4r __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4r __attribute__((ext_vector_type(4)));
typedef short s16x4r __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4r lds_s16x4r;

constexpr float kRowsLog2e = 1.4426950408889634f;
constexpr float kRowsLn2 = 0.6931471805599453f;
// The reference maximum is re-based only when a step's probabilities against
// it sum to more than this: every probability stays at most 2^8.
constexpr float kRowsRebase = 256.0f;

// Score forms (template argument of the kernels)
constexpr int kScoreCap = 1;    // bit 0: capped by a tanh
constexpr int kScoreSlope = 2;  // bit 1: falls with the distance

struct ScoreArgs {
    float scale_log2;     // softmax scale * log2(e)
    float cap_in;         // 2 log2(e) * softmax scale / cap
    float cap_out;        // cap * log2(e)
    const float *slopes;  // [hq] or NULL
};

// Key offset (within a 32-key block) of accumulator register v, lane half h.
__device__ __forceinline__ int rows_key_of_reg(int v, int h)
{
    return (v & 7) + 8 * h + 16 * (v >> 3);
}

// K row fed to MFMA row r: bits 2 and 3 swapped.
__device__ __forceinline__ int rows_perm(int r)
{
    return (r & ~12) | ((r & 4) << 1) | ((r & 8) >> 1);
}

__device__ __forceinline__ float rows_pair_max(float x)
{
    auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                              false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

__device__ __forceinline__ float rows_pair_sum(float x)
{
    auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                              false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// 16-byte chunk swizzles of the LDS tiles ([key][d] rows of 2 D bytes), which
// keep both operand reads free of bank conflicts.
template <int D>
__device__ __forceinline__ int rows_kswz(int r)
{
    return D == 128 ? (r & 15) : ((r >> 1) & 7);
}
template <int D>
__device__ __forceinline__ int rows_vswz(int r)
{
    return D == 128 ? 4 * (r & 3) : 4 * ((r >> 1) & 1);
}

// s_waitcnt vmcnt(N) alone (N < 64: low four bits, then two high ones).
template <int N>
__device__ __forceinline__ void rows_wait_copies()
{
    static_assert(N >= 0 && N < 64, "six bits of vmcnt");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | ((N >> 4) << 14));
    asm volatile("" ::: "memory");
}

// Log-sum-exps of rows whose scores grow with the distance count it from the
// first key: what the row's own distance from there, `past` keys, adds.
__device__ __forceinline__ float rows_lse_shift(float slope, int past)
{
    return slope < 0.f ? -slope * (float)past : 0.f;
}

// Score arguments of a call; false where a cap's factors leave fp32.
inline bool rows_score_args(ScoreArgs &a, float softmax_scale, float softcap, const float *slopes)
{
    a.scale_log2 = softmax_scale * kRowsLog2e;
    a.cap_in = softcap > 0.f ? 2.f * kRowsLog2e * (softmax_scale / softcap) : 0.f;
    a.cap_out = softcap * kRowsLog2e;
    a.slopes = slopes;
    return a.cap_in <= 3.0e38f;
}

// Largest cap: an error of 10 2^-24 of it is 6.1e-4 then.
constexpr float kRowsMaxCap = 1024.f;

// One wave's 32 rows.  NKB: 32-key blocks of a tile.
template <int D, int NKB, int SCORE>
struct RowBlock {
    static constexpr int ROW_BYTES = 2 * D;
    static constexpr int QK_STEPS = D / 16;
    static constexpr int D_BLOCKS = D / 32;

    bf16x8 qf[QK_STEPS];
    f32x16 oacc[D_BLOCKS];
    float m_ref;   // reference maximum, log2 domain
    float l_run;   // sum of this lane's probabilities
    uint32_t koff[QK_STEPS];
    uint32_t voff[D_BLOCKS];
    int half, col;

    __device__ __forceinline__ void init(int lane)
    {
        half = lane >> 5;
        col = lane & 31;
        const int krow = rows_perm(col);
#pragma unroll
        for (int s = 0; s < QK_STEPS; ++s)
            koff[s] = (uint32_t)(krow * ROW_BYTES + (((2 * s + half) ^ rows_kswz<D>(krow)) << 4));
        // transposed reads: in each group of 16 lanes, lane i addresses row
        // K0 + i / 4 at d = D0 + 4 (i % 4), and lane j receives rows
        // K0 .. K0 + 3 at d = D0 + j
        const int vrow = 8 * half + ((lane & 15) >> 2);
        const int tr_d = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
#pragma unroll
        for (int b = 0; b < D_BLOCKS; ++b) {
            const int d = 32 * b + tr_d;
            voff[b] = (uint32_t)(vrow * ROW_BYTES + (((d >> 3) ^ rows_vswz<D>(vrow)) << 4) +
                                 (d & 7) * 2);
        }
    }

    __device__ __forceinline__ void reset()
    {
#pragma unroll
        for (int b = 0; b < D_BLOCKS; ++b)
            oacc[b] = f32x16{};
        m_ref = -INFINITY;
        l_run = 0.f;
    }

    // The B operand of S^T = K Q^T from global memory: row points at this
    // lane's query row of D values.
    __device__ __forceinline__ void load_q(const uint16_t *row)
    {
#pragma unroll
        for (int s = 0; s < QK_STEPS; ++s)
            qf[s] = *reinterpret_cast<const bf16x8 *>(row + 16 * s + 8 * half);
    }

    // Raw products of one tile; hook(i) runs after MFMA i.
    template <typename F>
    __device__ __forceinline__ void products(const unsigned char *kt, f32x16 (&s)[NKB],
                                             F &&hook) const
    {
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb)
            s[kb] = f32x16{};
#pragma unroll
        for (int i = 0; i < QK_STEPS; ++i)
#pragma unroll
            for (int kb = 0; kb < NKB; ++kb) {
                const bf16x8 a =
                    *reinterpret_cast<const bf16x8 *>(kt + koff[i] + kb * 32 * ROW_BYTES);
                s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qf[i], s[kb], 0, 0, 0);
                hook(i * NKB + kb);
            }
    }
    __device__ __forceinline__ void products(const unsigned char *kt, f32x16 (&s)[NKB]) const
    {
        products(kt, s, [](int) {});
    }

    // Scores are held as values x of which the log2-domain score is
    // x factor + offset + slope (key - row): the products themselves, or for a
    // capped score -1 / (1 + e^(2 x / cap)), the factor then 2 cap and the offset
    // cap.  Factor, offset, bias and reference enter the exponent in one fused
    // multiply-add (two where there are slopes), and a key that drops out is
    // -inf either way.
    __device__ __forceinline__ void modify(f32x16 (&s)[NKB], const ScoreArgs &a) const
    {
        if constexpr ((SCORE & kScoreCap) != 0) {
#pragma unroll
            for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
                for (int v = 0; v < 16; ++v)
                    s[kb][v] = __builtin_amdgcn_rcpf(
                        -1.f - __builtin_amdgcn_exp2f(s[kb][v] * a.cap_in));
        }
    }
    __device__ __forceinline__ static float factor(const ScoreArgs &a)
    {
        return (SCORE & kScoreCap) != 0 ? 2.f * a.cap_out : a.scale_log2;
    }

    // Keys whose offset in the tile is above lim (this lane's row) drop out.
    __device__ __forceinline__ void mask_above(f32x16 (&s)[NKB], int lim) const
    {
        const int l = lim - 8 * half;
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
            for (int v = 0; v < 16; ++v)
                s[kb][v] = kb * 32 + rows_key_of_reg(v, 0) <= l ? s[kb][v] : -INFINITY;
    }

    // Probabilities against the lazily re-based reference, as the bf16 B
    // operand of PV.  They are first taken against the current reference: each
    // is >= 0, so where their sum is at most kRowsRebase none exceeds it.
    // Otherwise (also when no reference is set yet: the sum is then infinite
    // or NaN) the row maxima are taken and the accumulators rescaled.
    // dist0 = first key of the tile - the key that this lane's row counts
    // distances from; fresh: the first step, which has no reference on any lane;
    // weight(kb, v, p): what stands for the probability of register v's key in the
    // PV product (the sums take the probability itself).
    template <typename F>
    __device__ __forceinline__ void softmax(const f32x16 (&s)[NKB], const ScoreArgs &a,
                                            float slope_log2, int dist0, bf16x8 (&pf)[NKB][2],
                                            bool fresh, F &&weight)
    {
        const float f = factor(a);
        // distances below 2^24 are exact in fp32
        float base = (SCORE & kScoreCap) != 0 ? a.cap_out : 0.f;
        if constexpr ((SCORE & kScoreSlope) != 0)
            base = __builtin_fmaf(slope_log2, (float)(dist0 + 8 * half), base);
        auto score = [&](int kb, int v, float b) TA_INLINE -> float {
            if constexpr ((SCORE & kScoreSlope) != 0)
                b = __builtin_fmaf(slope_log2, (float)(kb * 32 + rows_key_of_reg(v, 0)), b);
            return __builtin_fmaf(s[kb][v], f, b);
        };
        auto exps = [&](float m) TA_INLINE -> float {
            const float b = base - m;
            float sum = 0.f;
#pragma unroll
            for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
                for (int s2 = 0; s2 < 2; ++s2) {
                    u32x4 packed;
#pragma unroll
                    for (int e = 0; e < 8; e += 2) {
                        typedef float f32x2r __attribute__((ext_vector_type(2)));
                        typedef __bf16 bf16x2r __attribute__((ext_vector_type(2)));
                        f32x2r t;
                        t[0] = __builtin_amdgcn_exp2f(score(kb, 8 * s2 + e, b));
                        t[1] = __builtin_amdgcn_exp2f(score(kb, 8 * s2 + e + 1, b));
                        sum = (kb | s2 | e) ? sum + t[0] : t[0];
                        sum += t[1];
                        t[0] = weight(kb, 8 * s2 + e, t[0]);
                        t[1] = weight(kb, 8 * s2 + e + 1, t[1]);
                        packed[e / 2] = __builtin_bit_cast(
                            uint32_t, __builtin_convertvector(t, bf16x2r));
                    }
                    pf[kb][s2] = __builtin_bit_cast(bf16x8, packed);
                }
            return sum;
        };
        float sum = INFINITY;
        if (!fresh)
            sum = exps(m_ref);
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(sum <= kRowsRebase)) != 0, 0)) {
            float mx = -INFINITY;
#pragma unroll
            for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
                for (int v = 0; v < 16; ++v)
                    mx = fmaxf(mx, score(kb, v, base));
            mx = rows_pair_max(mx);
            // only the rows that need it: a row's bits follow from its own
            // scores, not from the rows that share its wave
            const bool mine = rows_pair_max(sum <= kRowsRebase ? 0.f : 1.f) != 0.f;
            const float m_new = mine ? fmaxf(m_ref, mx) : m_ref;
            const float m_use = m_new == -INFINITY ? 0.f : m_new;
            const float alpha = __builtin_amdgcn_exp2f(m_ref - m_use);
            l_run *= alpha;
#pragma unroll
            for (int b = 0; b < D_BLOCKS; ++b)
#pragma unroll
                for (int v = 0; v < 16; ++v)
                    oacc[b][v] *= alpha;
            m_ref = m_new;
            sum = exps(m_use);
        }
        l_run += sum;
    }
    __device__ __forceinline__ void softmax(const f32x16 (&s)[NKB], const ScoreArgs &a,
                                            float slope_log2, int dist0, bf16x8 (&pf)[NKB][2],
                                            bool fresh)
    {
        softmax(s, a, slope_log2, dist0, pf, fresh, [](int, int, float p) { return p; });
    }

    __device__ __forceinline__ bf16x8 v_fragment(const unsigned char *vt, int kb, int s2,
                                                 int b) const
    {
        s16x4r part[2];
#pragma unroll
        for (int i2 = 0; i2 < 2; ++i2)
            part[i2] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (lds_s16x4r *)(vt + voff[b] + (kb * 32 + s2 * 16 + 4 * i2) * ROW_BYTES));
        return __builtin_bit_cast(bf16x8,
                                  __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7));
    }

    // O^T += V^T P^T for one tile; hook(i) runs after MFMA i.
    template <typename F>
    __device__ __forceinline__ void accumulate(const unsigned char *vt, const bf16x8 (&pf)[NKB][2],
                                               F &&hook)
    {
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
            for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
                for (int b = 0; b < D_BLOCKS; ++b) {
                    oacc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                        v_fragment(vt, kb, s2, b), pf[kb][s2], oacc[b], 0, 0, 0);
                    hook((kb * 2 + s2) * D_BLOCKS + b);
                }
    }
    __device__ __forceinline__ void accumulate(const unsigned char *vt, const bf16x8 (&pf)[NKB][2])
    {
        accumulate(vt, pf, [](int) {});
    }

    // products() of one tile (QK) and then accumulate() of another (PV), each
    // fragment read AHEAD matrix instructions before its own, in this order as it
    // stands: where registers are scarce the scheduler undoes the one that schedule()
    // asks for, and every matrix instruction waits for its read.
    template <bool QK, bool PV, int AHEAD = 4>
    __device__ __forceinline__ void in_order(const unsigned char *kt, const unsigned char *vt,
                                             f32x16 (&s)[NKB], const bf16x8 (&pf)[NKB][2])
    {
        constexpr int NQ = QK ? NKB * QK_STEPS : 0, N = NQ + (PV ? NKB * 2 * D_BLOCKS : 0);
        auto read = [&](int i) TA_INLINE -> bf16x8 {
            if (i < NQ)
                return *reinterpret_cast<const bf16x8 *>(kt + koff[i / NKB] +
                                                         i % NKB * 32 * ROW_BYTES);
            const int j = i - NQ;
            return v_fragment(vt, j / (2 * D_BLOCKS), j / D_BLOCKS % 2, j % D_BLOCKS);
        };
        __builtin_amdgcn_sched_barrier(0);
        bf16x8 ahead[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
            ahead[i] = read(i);
        if constexpr (QK)
#pragma unroll
            for (int kb = 0; kb < NKB; ++kb)
                s[kb] = f32x16{};
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (i < NQ) {
                s[i % NKB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                    ahead[i % AHEAD], qf[i / NKB], s[i % NKB], 0, 0, 0);
            } else {
                const int j = i - NQ, b = j % D_BLOCKS;
                oacc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                    ahead[i % AHEAD], pf[j / (2 * D_BLOCKS)][j / D_BLOCKS % 2], oacc[b], 0, 0, 0);
            }
            if (i + AHEAD < N)
                ahead[i % AHEAD] = read(i + AHEAD);
            __builtin_amdgcn_sched_barrier(0);
        }
    }

    // Whether a tile holds an infinite or NaN value (this wave looks at part
    // `part` of `parts`).  In a masked step rows give keys probability zero that
    // other rows keep, and zero times such a value must not reach them:
    // accumulate_by_key then takes the place of accumulate.
    __device__ __forceinline__ static bool odd_values(const unsigned char *vt, int lane, int part,
                                                      int parts)
    {
        constexpr int BYTES = NKB * 32 * ROW_BYTES;
        uint32_t carry = 0;
        for (int i = part; i < BYTES / 1024; i += parts) {
            const u32x4 w = *reinterpret_cast<const u32x4 *>(vt + i * 1024 + lane * 16);
#pragma unroll
            for (int e = 0; e < 4; ++e)  // an exponent of all ones carries into the sign bit
                carry |= (w[e] & 0x7f807f80u) + 0x00800080u;
        }
        return __builtin_amdgcn_ballot_w64((carry & 0x80008000u) != 0) != 0;
    }

    // What stands in pf for this lane's row at key j of a tile, and whether the row
    // keeps that key (whose score x, as the mask left it, is then not -inf).
    __device__ __forceinline__ bool weight_of_key(int j, const f32x16 (&x)[NKB],
                                                  const bf16x8 (&pf)[NKB][2], float &p) const
    {
        typedef uint16_t u16x8r __attribute__((ext_vector_type(8)));
        // key j: block j / 32, element (j / 16 & 1, j & 7) of half j / 8 & 1
        float mine = 0.f, kept = 0.f;
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
            for (int s2 = 0; s2 < 2; ++s2) {
                const u16x8r pb = __builtin_bit_cast(u16x8r, pf[kb][s2]);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const bool on = kb * 32 + s2 * 16 + 8 * half + e == j;
                    mine = on ? __uint_as_float((uint32_t)pb[e] << 16) : mine;
                    kept = on && x[kb][8 * s2 + e] != -INFINITY ? 1.f : kept;
                }
            }
        p = rows_pair_sum(mine);
        return rows_pair_sum(kept) != 0.f;
    }

    // accumulate() key by key, each only to the rows that keep it.
    __device__ __forceinline__ void accumulate_by_key(const unsigned char *vt,
                                                      const f32x16 (&x)[NKB],
                                                      const bf16x8 (&pf)[NKB][2])
    {
        typedef uint16_t u16x4r __attribute__((ext_vector_type(4)));
#pragma unroll 1
        for (int j = 0; j < NKB * 32; ++j) {
            float p;
            const bool keeps = weight_of_key(j, x, pf, p);
            const unsigned char *row = vt + j * ROW_BYTES;
#pragma unroll
            for (int b = 0; b < D_BLOCKS; ++b)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    // accumulators 4 c .. 4 c + 3: d = 32 b + 8 c + 4 half ..
                    const u16x4r v = *reinterpret_cast<const u16x4r *>(
                        row + (((4 * b + c) ^ rows_vswz<D>(j)) << 4) + 8 * half);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        oacc[b][4 * c + e] +=
                            keeps ? p * __uint_as_float((uint32_t)v[e] << 16) : 0.f;
                }
        }
    }

    // Order of the LDS reads and MFMAs issued since the last scheduling region
    // began: products() when QK, then accumulate() when PV.  MFMA i of products
    // needs one read (a K fragment), one of accumulate two; the reads of MFMA i +
    // AHEAD go out just before MFMA i, so that their latency (over a hundred
    // cycles under load, four MFMAs) is covered.
    template <bool QK, bool PV>
    __device__ __forceinline__ static void schedule()
    {
        constexpr int NQ = QK ? NKB * QK_STEPS : 0, N = NQ + (PV ? NKB * 2 * D_BLOCKS : 0);
        constexpr int AHEAD = N < 6 ? N : 6;
        constexpr int first = AHEAD <= NQ ? AHEAD : NQ + 2 * (AHEAD - NQ);
        __builtin_amdgcn_sched_group_barrier(kSchedDsRead, first, 0);
        schedule_from<NQ, N, AHEAD, 0>();
    }
    template <int NQ, int N, int AHEAD, int I>
    __device__ __forceinline__ static void schedule_from()
    {
        if constexpr (I < N) {
            __builtin_amdgcn_sched_group_barrier(kSchedMfma, 1, 0);
            if constexpr (I + AHEAD < N)
                __builtin_amdgcn_sched_group_barrier(kSchedDsRead, I + AHEAD < NQ ? 1 : 2, 0);
            schedule_from<NQ, N, AHEAD, I + 1>();
        }
    }

    // 1 / sum and the natural log-sum-exp of the row (0 and -inf: no key; a
    // NaN sum stays visible).
    __device__ __forceinline__ void finish(float &inv, float &lse) const
    {
        const float l = rows_pair_sum(l_run);
        inv = l == 0.f ? 0.f : 1.f / l;
        lse = l == 0.f ? -INFINITY : (m_ref + __log2f(l)) * kRowsLn2;
    }
};

}  // namespace triattn
