// Prefill attention with modified scores (capped by a tanh, falling with the
// distance) over the schedules of the forward passes: Triangle, dense causal
// and block-sparse.
//
// A workgroup of four or eight waves takes as many row blocks (32 rows of one
// head) of a schedule item, dealt out head first, over K/V tiles of 64 keys in
// LDS.  What bounds it: the two products take a wave 32 matrix instructions of 32
// cycles a step.  A capped score takes two exp2, a reciprocal and five plain
// instructions: 1535 cycles of the vector unit a step by its counter, more than the
// matrix cores' 1024.  The 16384-token causal layer (32 heads over 8, d = 128) runs
// at 2050 cycles a wave and step, 2.20 ms, 998 TFLOP/s, vector units 75 % and matrix
// cores 50 % busy.  Slopes add one operation to a plain score: packed 42000 tokens
// at window 2048 in 1.39 ms, 1056 TFLOP/s, matrix cores 56 % and vector units 54 %
// busy.  A slope below zero makes every step outgrow the softmax reference, and
// rescale: 16384 tokens 2.71 ms, and 1.71 with slopes above zero.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "triattn_device.h"
#include "triattn_internal.h"
#include "triattn_rows.h"

namespace triattn {
namespace {

constexpr int kJoinThreads = 256;
constexpr int kKeys = 64;           // keys of a step
constexpr int kListSteps = 2048;    // steps of a list item held in LDS

struct ScoredArgs {
    const uint16_t *q, *k, *v;
    void *o;
    float *lse;
    const int32_t *sched;
    float *part_o, *part_lse;  // [partial rows, hq (, D)]
    ScoreArgs score;
    int64_t total_tokens, list_base, list_words;
    int32_t kind, tile, hq, hkv, group, sink, window;
    int32_t n_items, n_merges, n_partial_rows;
    int32_t subtiles;  // workgroups per item and kv head
    int32_t o_f32;
};

// The steps that one workgroup's rows can reach: two runs of 64-key steps, a
// then b, or a list.
struct Runs {
    int a_lo, a_hi, b_lo, b_hi;
};

// Drops the steps in which none of the rows wr0 .. wr1 keeps a key: past the
// last row, and for streaming rows between the sink and the first row's window.
__device__ __forceinline__ Runs reach(Runs r, bool stream, int sink, int window, int wr0, int wr1)
{
    if (stream) {
        const int band = max(wr0 - window + 1, 0) / kKeys;
        // (a sink past the rows is one of all their keys; its own length may be
        // any number of 32 bits)
        const int sinks = (min(sink, wr1 + 1) + kKeys - 1) / kKeys;
        if (r.b_hi > r.b_lo) {
            r.a_hi = max(min(r.a_hi, sinks), r.a_lo);
            r.b_lo = min(max(r.b_lo, band), r.b_hi);
        } else if (band > sinks || sink == 0) {
            r.b_hi = r.a_hi;
            r.b_lo = min(max(r.a_lo, band), r.a_hi);
            r.a_hi = max(min(r.a_hi, sink == 0 ? r.a_lo : sinks), r.a_lo);
        }
    }
    const int end = wr1 / kKeys + 1;
    r.a_hi = max(min(r.a_hi, end), r.a_lo);
    r.b_hi = max(min(r.b_hi, end), r.b_lo);
    return r;
}

template <int D, int SCORE, bool LIST, int NW>
__global__ __launch_bounds__(NW * 64, D == 64 ? 3 : 2) void scored_attn_kernel(ScoredArgs a)
{
    static_assert(NW == 4 || D == 128, "eight waves at d = 128 only");
    constexpr int kThreads = NW * 64;
    constexpr int ROW_BYTES = 2 * D;
    constexpr int CHUNKS = D / 8;
    constexpr int TILE_BYTES = kKeys * ROW_BYTES;
    constexpr int STAGE_BYTES = 2 * TILE_BYTES;  // K tile, then V tile
    constexpr int COPY_ROWS = 1024 / ROW_BYTES;  // keys of a 1 KB copy
    constexpr int COPIES = TILE_BYTES / 1024 / 4;  // of a copying wave, for K and again for V
    constexpr int D_BLOCKS = D / 32;

    __shared__ __attribute__((aligned(1024))) unsigned char smem[2 * STAGE_BYTES];
    __shared__ int32_t s_key[LIST ? kListSteps : 1];

    const int32_t *sched = a.sched;
    int bid = blockIdx.x;
    const int g = bid % a.hkv;
    bid /= a.hkv;
    const int sub = bid % a.subtiles;
    // (causal and block-sparse schedules list the longest items first)
    const int item = bid / a.subtiles;
    const int32_t *it = sched + kHdrWords + (int64_t)item * kItemWords;
    const int64_t seq_off = it[I_SEQ_OFF];
    const int32_t seq_len = it[I_SEQ_LEN];
    const int32_t r0 = it[I_R0], r1 = it[I_R1];
    const int32_t ka0 = it[I_KA0], ka1 = it[I_KA1], kb0 = it[I_KB0], kb1 = it[I_KB1];
    const int32_t mode = it[I_MODE], part_base = it[I_PART_BASE];
    const bool list = LIST && mode == kModeCausalList;
    const int64_t sched_total =
        (int64_t)(uint32_t)sched[H_TOTAL_LO] | ((int64_t)sched[H_TOTAL_HI] << 32);
    const bool bad =
        (sched[H_MAGIC] != TA_SCHEDULE_MAGIC) | (sched[H_VERSION] != TA_SCHEDULE_VERSION) |
        (sched[H_KIND] != a.kind) | (sched_total != a.total_tokens) |
        (sched[H_ITEMS] != a.n_items) | (sched[H_TILE] != a.tile) |
        (LIST & (sched[H_WINDOW] != a.list_words)) | (seq_off < 0) | (seq_len < 0) |
        (seq_off + seq_len > a.total_tokens) | (r0 < 0) | (r1 > seq_len) | (r0 >= r1) |
        (r1 - r0 > a.tile) | (ka0 < 0) | (kb0 < 0) | (kb1 < kb0) |
        (mode != kModeStreaming && mode != kModeCausal && !list) |
        (list ? (ka1 < 0) | (kb1 != kb0) | ((int64_t)ka0 + ka1 > a.list_words) : ka1 < ka0) |
        (part_base >= 0 && (int64_t)part_base + (r1 - r0) > a.n_partial_rows);
    if (bad) {
        poison_outputs(a.o, a.o_f32, a.lse, a.total_tokens, a.hq, D, blockIdx.x, gridDim.x);
        poison_item_rows(a.o, a.o_f32, a.lse, a.part_o, a.part_lse, a.total_tokens, a.hq, D,
                         a.n_partial_rows, a.tile, seq_off, r0, r1, part_base);
        return;
    }
    const int max_ktile = (seq_len - 1) / a.tile;
    const bool stream = mode == kModeStreaming;

    const int tid = threadIdx.x;
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // row block b: head b % group, rows 32 (b / group) on
    const int b0 = NW * sub;
    const int wr0 = r0 + 32 * (b0 / a.group);
    if (wr0 >= r1)
        return;  // ragged q-tile: nothing for this workgroup
    const int wr1 = min(r0 + 32 * ((b0 + NW - 1) / a.group + 1), r1) - 1;
    const int head = g * a.group + (b0 + wave) % a.group;
    const int row_base = r0 + 32 * ((b0 + wave) / a.group);
    const bool active = row_base < r1;
    const int row_hi = min(row_base + 31, r1 - 1);

    RowBlock<D, 2, SCORE> rb;
    rb.init(lane);
    const int row = min(row_base + rb.col, r1 - 1);
    rb.load_q(a.q + ((seq_off + row) * a.hq + head) * (int64_t)D);
    float slope = 0.f;
    if constexpr ((SCORE & kScoreSlope) != 0)
        slope = a.score.slopes[head] * kRowsLog2e;
    // Where distances are taken from, so that they are short at the keys that
    // weigh most and round to little there: the row where scores fall with the
    // distance, its first key where they grow with it (of all rows that have
    // partials or a sink the sequence's first; the log-sum-exp gets what the row
    // is past that at its very end).
    int from = row;
    if constexpr ((SCORE & kScoreSlope) != 0)
        if (slope < 0.f)
            from = stream && a.sink == 0 ? max(0, row - a.window + 1) : 0;

    // steps
    const int tps = a.tile / kKeys;
    Runs runs{ka0 * tps, ka1 * tps, kb0 * tps, kb1 * tps};
    int n;
    const int32_t *tiles = sched + a.list_base + (list ? ka0 : 0);
    auto listed = [&](int s) TA_INLINE -> int {
        return min(max(tiles[s / tps], 0), max_ktile) * a.tile + (s % tps) * kKeys;
    };
    if (list) {
        n = ka1 * tps;
        for (int s = tid; s < min(n, kListSteps); s += kThreads)
            s_key[s] = listed(s);
        __syncthreads();
    } else {
        runs = reach(runs, stream, a.sink, a.window, wr0, wr1);
        n = runs.a_hi - runs.a_lo + runs.b_hi - runs.b_lo;
    }
    // Step i of the pass.  Where scores fall with the distance the steps run
    // from the last key to the first: a row's largest scores come first, and
    // its reference stands (in the other order each step's outgrow it, and
    // nearly every step of a steep head rescales the accumulators).
    auto step_key = [&](int i) TA_INLINE -> int {
        const int s = (SCORE & kScoreSlope) != 0 ? n - 1 - i : i;
        if (list)
            return __builtin_amdgcn_readfirstlane(s < kListSteps ? s_key[s] : listed(s));
        const int na = runs.a_hi - runs.a_lo;
        return (s < na ? runs.a_lo + s : runs.b_lo + s - na) * kKeys;
    };
    if (list)  // listed tiles increase: only the last may pass the rows
        while (n > 0 && listed(n - 1) > wr1)
            --n;

    // copies: of the first four waves, wave w takes 1 KB blocks w COPIES .. of a
    // tile.  The swizzle of block i's rows is that of block 0's with the bits of
    // i COPY_ROWS flipped (K; V's does not depend on them).
    const uint32_t smem_addr =
        (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)smem;
    const uint32_t pitch = (uint32_t)(a.hkv * ROW_BYTES);
    const uint16_t *kbase = a.k + (seq_off * a.hkv + g) * (int64_t)D;
    const uint16_t *vbase = a.v + (seq_off * a.hkv + g) * (int64_t)D;
    const int dma_row = wave * COPIES * COPY_ROWS + lane / CHUNKS;
    const uint32_t dma_off = __umul24((uint32_t)dma_row, pitch);
    const uint32_t kswz = (uint32_t)(((lane % CHUNKS) ^ rows_kswz<D>(dma_row)) << 4);
    const uint32_t vswz = (uint32_t)(((lane % CHUNKS) ^ rows_vswz<D>(dma_row)) << 4);
    static_assert((COPIES & (COPIES - 1)) == 0 && COPIES <= 4, "blocks of a wave differ in bits");
    // Where a step's keys are.  Rows past the sequence repeat its last one; no
    // row keeps them.
    struct Place {
        int key0;
        bool masked;   // some row of the workgroup drops keys of it
        uint32_t lim;  // byte offset of the tile's last row
        int64_t off;   // elements to its first row
    };
    auto place = [&](int i) TA_INLINE -> Place {
        Place x;
        x.key0 = step_key(i);
        x.masked = (x.key0 + kKeys - 1 > wr0) |
                   (stream & (x.key0 + kKeys - 1 >= a.sink) & (wr1 - x.key0 >= a.window));
        const int first = min(x.key0, seq_len - 1);
        x.lim = (uint32_t)min(seq_len - 1 - first, kKeys - 1) * pitch;
        x.off = (int64_t)first * a.hkv * D;
        return x;
    };
    // block i of this wave, K or V
    auto copy_block = [&](const Place &x, int i, int stage, auto is_v) TA_INLINE {
        constexpr bool V = decltype(is_v)::value;
        const uint32_t swz = V ? vswz : kswz ^ (uint32_t)(rows_kswz<D>(i * COPY_ROWS) << 4);
        copy_to_lds16((V ? vbase : kbase) + x.off,
                      min(dma_off + (uint32_t)(i * COPY_ROWS) * pitch, x.lim) + swz,
                      smem_addr + stage * STAGE_BYTES + (V ? TILE_BYTES : 0) +
                          (wave * COPIES + i) * 1024);
    };
    auto copy_k = [&](const Place &x, int stage) TA_INLINE {
#pragma unroll
        for (int i = 0; i < COPIES; ++i)
            copy_block(x, i, stage, std::false_type{});
    };
    auto copy_v = [&](const Place &x, int stage) TA_INLINE {
#pragma unroll
        for (int i = 0; i < COPIES; ++i)
            copy_block(x, i, stage, std::true_type{});
    };
    auto end_phase = [&](bool copies) TA_INLINE {
        __builtin_amdgcn_sched_barrier(0);
        if (copies)
            rows_wait_copies<0>();
        barrier_no_fence();
        __builtin_amdgcn_sched_barrier(0);
    };

    f32x16 s[2];
    bf16x8 p[2][2];
    bool fresh, odd;
    // Keys that this wave's rows drop (three comparisons a score only where a
    // step holds more than one of the edges).
    auto mask = [&](int key0) TA_INLINE {
        const bool diagonal = key0 + kKeys - 1 > row_base;
        const bool edge = stream & (key0 + kKeys - 1 >= a.sink) & (row_hi - key0 >= a.window);
        if (!edge) {
            if (diagonal)
                rb.mask_above(s, row - key0);
            return;
        }
        const int lim = row - key0 - 8 * rb.half;
        const int far = lim - a.window;                 // in the window: offset > far
        const int sinks = a.sink - key0 - 8 * rb.half;  // in the sink: offset < sinks
        auto keep = [&](auto &&test) TA_INLINE {
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int v = 0; v < 16; ++v)
                    s[kb][v] = test(kb * 32 + rows_key_of_reg(v, 0)) ? s[kb][v] : -INFINITY;
        };
        if (!diagonal && key0 >= a.sink)
            keep([&](int off) TA_INLINE { return off > far; });
        else if (key0 + kKeys - 1 <= row_base - a.window)
            keep([&](int off) TA_INLINE { return off < sinks; });
        else
            keep([&](int off) TA_INLINE { return (off <= lim) & ((off > far) | (off < sinks)); });
    };
    // X(j): the scores of step j to probabilities
    auto softmax = [&](const Place &x) TA_INLINE {
        rb.modify(s, a.score);
        if (__builtin_expect(x.masked, 0)) {
            asm volatile("");  // a branch: most steps have no mask
            mask(x.key0);
        }
        rb.softmax(s, a.score, slope, x.key0 - from, p, fresh);
        fresh = false;
    };
    // The values of a masked step, each wave its part of the tile (apart from
    // the common path).
    auto look = [&](const Place &x, const unsigned char *vt) TA_INLINE {
        if (__builtin_expect(x.masked, 0)) {
            asm volatile("");
            odd |= rb.odd_values(vt, lane, wave, NW);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    // O += V P of the step whose probabilities p holds
    auto values = [&](const Place &x, const unsigned char *vt) TA_INLINE {
        look(x, vt);
        rb.accumulate(vt, p);
        rb.template schedule<false, true>();
        __builtin_amdgcn_sched_barrier(0);
    };
    auto products = [&](const unsigned char *kt) TA_INLINE {
        __builtin_amdgcn_sched_barrier(0);
        rb.products(kt, s);
        rb.template schedule<true, false>();
        __builtin_amdgcn_sched_barrier(0);
    };
    using Stage0 = std::integral_constant<int, 0>;
    using Stage1 = std::integral_constant<int, 1>;

    // One pass over the steps, every wave in the same one; `odd` tells
    // whether a masked step holds infinite or NaN values.
    auto together = [&]() TA_INLINE {
        Place now = place(0);
        copy_k(now, 0);
        copy_v(now, 0);
        auto step = [&](int i, auto stage) TA_INLINE {
            constexpr int ST = decltype(stage)::value;
            // this step's tile has landed for every wave, and every wave is
            // done with the other stage
            end_phase(true);
            const Place next = place(min(i + 1, n - 1));
            if (i + 1 < n) {
                copy_k(next, 1 - ST);
                copy_v(next, 1 - ST);
            }
            const unsigned char *kt = smem + ST * STAGE_BYTES;
            products(kt);
            softmax(now);
            values(now, kt + TILE_BYTES);
            now = next;
        };
        int i = 0;
        for (; i + 1 < n; i += 2) {
            step(i, Stage0{});
            step(i + 1, Stage1{});
        }
        if (i < n)
            step(i, Stage0{});
    };
    // The pass that keeps infinite and NaN values in masked steps from the
    // rows that do not keep their keys.
    auto careful = [&]() TA_INLINE {
        for (int i = 0; i < n; ++i) {
            const Place now = place(i);
            if (wave < 4) {
                copy_k(now, 0);
                copy_v(now, 0);
            }
            end_phase(true);
            products(smem);
            softmax(now);
            rb.accumulate_by_key(smem + TILE_BYTES, s, p);
            end_phase(false);
        }
    };
    // The same in two groups of four waves, one wave of each on a SIMD, in
    // turns: M(j) = {S(j) = K(j) Q^T, O += V(j - 1) P(j - 1)} on the matrix
    // cores beside the other group's X(j) on the vector units.  Group 0 runs
    // M(j) in phase 2 j and X(j) in phase 2 j + 1, group 1 X(j - 1) in phase 2 j
    // and M(j) in phase 2 j + 1.  Stage j & 1 holds K(j) and V(j - 1) in these
    // two phases; group 0 copies K(j + 1) and V(j) into the other one, last read
    // in phase 2 j - 1, spread over the MFMAs of M(j): issue slots that are free
    // there.
    auto in_turns = [&]() TA_INLINE {
        constexpr int NQ = 2 * (D / 16);        // MFMAs of products()
        constexpr int SLOTS = NQ + 4 * (D / 32);  // and of accumulate()
        constexpr int STRIDE = SLOTS / (2 * COPIES);
        Place prev, now = place(0), next = place(min(1, n - 1));
        auto matrix = [&](auto stage, auto &&hook) TA_INLINE {
            const unsigned char *kt = smem + decltype(stage)::value * STAGE_BYTES;
            look(prev, kt + TILE_BYTES);
            __builtin_amdgcn_s_setprio(1);
            __builtin_amdgcn_sched_barrier(0);
            rb.products(kt, s, hook);
            rb.accumulate(kt + TILE_BYTES, p, [&](int i) TA_INLINE { hook(NQ + i); });
            rb.template schedule<true, true>();
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(0);
        };
        auto advance = [&](int j) TA_INLINE {  // to step j
            prev = now;
            now = next;
            next = place(min(j + 1, n - 1));
        };
        int j = 1;
        if (wave < 4) {
            copy_k(now, 0);
            end_phase(true);
            copy_k(next, 1);
            copy_v(now, 1);
            products(smem);
            end_phase(false);
            softmax(now);
            end_phase(true);
            auto step = [&](int j, auto stage) TA_INLINE {
                constexpr int OTHER = 1 - decltype(stage)::value;
                advance(j);
                matrix(stage, [&](int i) TA_INLINE {
                    if (i % STRIDE == STRIDE - 1) {
                        const int c = i / STRIDE;
                        if (c < COPIES)
                            copy_block(next, c, OTHER, std::false_type{});
                        else if (c < 2 * COPIES)
                            copy_block(now, c - COPIES, OTHER, std::true_type{});
                    }
                });
                end_phase(false);
                softmax(now);
                end_phase(true);
            };
            for (; j + 1 < n; j += 2) {
                step(j, Stage1{});
                step(j + 1, Stage0{});
            }
            if (j < n)
                step(j, Stage1{});
            values(now, smem + (n & 1) * STAGE_BYTES + TILE_BYTES);
            end_phase(false);
            end_phase(false);
        } else {
            end_phase(false);
            end_phase(false);
            products(smem);
            end_phase(false);
            auto step = [&](int j, auto stage) TA_INLINE {
                softmax(now);
                end_phase(false);
                advance(j);
                matrix(stage, [](int) {});
                end_phase(false);
            };
            for (; j + 1 < n; j += 2) {
                step(j, Stage1{});
                step(j + 1, Stage0{});
            }
            if (j < n)
                step(j, Stage1{});
            softmax(now);
            end_phase(false);
            values(now, smem + (n & 1) * STAGE_BYTES + TILE_BYTES);
            end_phase(false);
        }
    };
    auto start = [&]() TA_INLINE {
        fresh = true;
        odd = false;
        rb.reset();
    };
    start();
    if (n > 0) {
        if constexpr (NW == 8)
            in_turns();
        else
            together();
        if (__builtin_expect(__syncthreads_or(odd), 0)) {
            start();
            careful();
        }
    }
    if (!active || row_base + rb.col >= r1)
        return;
    float inv, lse;
    rb.finish(inv, lse);
    const int64_t tok = seq_off + row;
    const int64_t prow = (int64_t)part_base + (row - r0);
#pragma unroll
    for (int b = 0; b < D_BLOCKS; ++b)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            f32x4r x;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                x[e] = rb.oacc[b][4 * c + e] * inv;
            const int d = 32 * b + 8 * c + 4 * rb.half;
            if (part_base >= 0)
                *reinterpret_cast<f32x4r *>(a.part_o + (prow * a.hq + head) * D + d) = x;
            else if (a.o_f32)
                *reinterpret_cast<f32x4r *>(static_cast<float *>(a.o) +
                                            (tok * a.hq + head) * D + d) = x;
            else
                *reinterpret_cast<bf16x4r *>(static_cast<__bf16 *>(a.o) +
                                             (tok * a.hq + head) * D + d) =
                    __builtin_convertvector(x, bf16x4r);
        }
    if (rb.half == 0) {
        if (part_base >= 0) {
            a.part_lse[prow * a.hq + head] = lse;
        } else if (a.lse) {
            if constexpr ((SCORE & kScoreSlope) != 0)
                lse += rows_lse_shift(a.score.slopes[head], row - from);
            a.lse[(int64_t)head * a.total_tokens + tok] = lse;
        }
    }
}

// Joins the partials of the schedule's split q-tiles, a wave to a (row, head):
// O = sum_c w_c O_c / sum_c w_c with w_c = exp(LSE_c - max_c LSE_c).
template <int D>
__device__ __forceinline__ void join_item(const ScoredArgs &a, int m)
{
    constexpr int PER = D / 64, kWaves = kJoinThreads / 64;
    const int32_t *sched = a.sched;
    const int32_t *x = sched + kHdrWords + (int64_t)a.n_items * kItemWords +
                       (int64_t)m * kMergeWords;
    const int64_t seq_off = x[M_SEQ_OFF];
    const int32_t r0 = x[M_R0], r1 = x[M_R1], ns = x[M_SPLITS], pb = x[M_PART_BASE];
    const int rows = r1 - r0;
    const int64_t sched_total =
        (int64_t)(uint32_t)sched[H_TOTAL_LO] | ((int64_t)sched[H_TOTAL_HI] << 32);
    if ((sched[H_MAGIC] != TA_SCHEDULE_MAGIC) | (sched[H_VERSION] != TA_SCHEDULE_VERSION) |
        (sched[H_KIND] != a.kind) | (sched_total != a.total_tokens) |
        (sched[H_ITEMS] != a.n_items) | (sched[H_TILE] != a.tile) | (rows < 1) |
        (rows > a.tile) | (ns < 1) | (pb < 0) |
        ((int64_t)pb + (int64_t)ns * rows > a.n_partial_rows) | (seq_off < 0) | (r0 < 0) |
        (seq_off + r1 > a.total_tokens)) {
        poison_outputs(a.o, a.o_f32, a.lse, a.total_tokens, a.hq, D,
                       (int64_t)blockIdx.y * gridDim.x + blockIdx.x,
                       (int64_t)gridDim.x * gridDim.y);
        poison_item_rows(a.o, a.o_f32, a.lse, nullptr, nullptr, a.total_tokens, a.hq, D, 0, a.tile,
                         seq_off, r0, r1, -1);
        return;
    }
    const int lane = threadIdx.x & 63;
    const int w = (int)blockIdx.x * kWaves + (threadIdx.x >> 6);
    const int head = w % a.hq, r = w / a.hq;
    if (r >= rows)
        return;
    auto at = [&](int c) TA_INLINE -> int64_t {
        return ((int64_t)pb + (int64_t)c * rows + r) * a.hq + head;
    };
    float mx = -INFINITY;
    for (int c = lane; c < ns; c += 64)
        mx = fmaxf(mx, a.part_lse[at(c)]);
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1)
        mx = fmaxf(mx, __shfl_xor(mx, o));
    const float m_use = mx == -INFINITY ? 0.f : mx;
    float acc[PER] = {}, den = 0.f;
    constexpr int UNROLL = 8;
    for (int c = 0; c < ns; c += UNROLL) {
        float y[UNROLL][PER], l[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const int64_t p = at(min(c + u, ns - 1));
            l[u] = a.part_lse[p];
#pragma unroll
            for (int e = 0; e < PER; ++e)
                y[u][e] = a.part_o[p * D + PER * lane + e];
        }
#pragma unroll
        for (int u = 0; u < UNROLL; ++u)
            if (c + u < ns) {
                const float f = __expf(l[u] - m_use);
                den += f;
#pragma unroll
                for (int e = 0; e < PER; ++e)
                    acc[e] += f * y[u][e];
            }
    }
    const float inv = den == 0.f ? 0.f : 1.f / den;
    const int64_t tok = seq_off + r0 + r;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        const int64_t i = (tok * a.hq + head) * D + PER * lane + e;
        if (a.o_f32)
            static_cast<float *>(a.o)[i] = acc[e] * inv;
        else
            static_cast<__bf16 *>(a.o)[i] = (__bf16)(acc[e] * inv);
    }
    if (a.lse && lane == 0)
        a.lse[(int64_t)head * a.total_tokens + tok] =
            den == 0.f ? -INFINITY
                       : m_use + __logf(den) +
                             (a.score.slopes ? rows_lse_shift(a.score.slopes[head], r0 + r) : 0.f);
}

// Grid: x covers the tile * hq (row, head) waves of a merge item, y the merge
// items, in turn where there are more than it holds.
template <int D>
__global__ __launch_bounds__(kJoinThreads) void scored_join_kernel(ScoredArgs a)
{
    for (int m = blockIdx.y; m < a.n_merges; m += gridDim.y)
        join_item<D>(a, m);
}

template <int D, bool LIST, int NW>
void launch_scored(int score, dim3 grid, hipStream_t s, const ScoredArgs &a)
{
    const dim3 threads(NW * 64);
    switch (score) {
    case 1: hipLaunchKernelGGL((scored_attn_kernel<D, 1, LIST, NW>), grid, threads, 0, s, a); break;
    case 2: hipLaunchKernelGGL((scored_attn_kernel<D, 2, LIST, NW>), grid, threads, 0, s, a); break;
    default: hipLaunchKernelGGL((scored_attn_kernel<D, 3, LIST, NW>), grid, threads, 0, s, a); break;
    }
}

template <int D, int NW>
void launch_scored(bool list, int score, dim3 grid, hipStream_t s, const ScoredArgs &a)
{
    if (list)
        launch_scored<D, true, NW>(score, grid, s, a);
    else
        launch_scored<D, false, NW>(score, grid, s, a);
}

}  // namespace
}  // namespace triattn

using namespace triattn;

extern "C" ta_status scored_attn_fwd(const void *q, const void *k, const void *v, void *o,
                                     int32_t o_dtype, float *lse, const int32_t *sched_dev,
                                     const ta_schedule_info *info, int64_t total_tokens,
                                     int32_t hq, int32_t hkv, int32_t head_dim,
                                     float softmax_scale, float softcap, const float *slopes,
                                     void *workspace, size_t workspace_bytes, void *stream)
{
    clear_error();
    const char *fn = "scored_attn_fwd";
    if (!info)
        return fail(TA_ERR_INVALID_ARG, "%s: info is NULL", fn);
    if (info->version != TA_SCHEDULE_VERSION)
        return fail(TA_ERR_SCHEDULE_MISMATCH, "%s: schedule version %d != %d", fn, info->version,
                    TA_SCHEDULE_VERSION);
    if (info->kind != TA_KIND_TRIANGLE && info->kind != TA_KIND_CAUSAL &&
        info->kind != TA_KIND_BLOCKSPARSE)
        return fail(TA_ERR_SCHEDULE_MISMATCH, "%s: schedule kind %d", fn, info->kind);
    if (total_tokens < 0)
        return fail(TA_ERR_INVALID_ARG, "%s: total_tokens < 0", fn);
    if (info->total_tokens != total_tokens)
        return fail(TA_ERR_SCHEDULE_MISMATCH, "%s: schedule built for %lld tokens, call has %lld",
                    fn, (long long)info->total_tokens, (long long)total_tokens);
    if (hq <= 0 || hkv <= 0)
        return fail(TA_ERR_INVALID_ARG, "%s: hq and hkv must be positive", fn);
    if (hq % hkv != 0)
        return fail(TA_ERR_INVALID_ARG, "%s: hq %d not a multiple of hkv %d", fn, hq, hkv);
    if (hq / hkv > 8)
        return fail(TA_ERR_UNSUPPORTED, "%s: GQA group %d > 8", fn, hq / hkv);
    if (head_dim != 64 && head_dim != 128)
        return fail(TA_ERR_UNSUPPORTED, "%s: head_dim %d not in {64, 128}", fn, head_dim);
    if (info->tile != 64 && info->tile != 128)
        return fail(TA_ERR_UNSUPPORTED, "%s: tile %d not in {64, 128}", fn, info->tile);
    if (o_dtype != TA_OUT_BF16 && o_dtype != TA_OUT_F32)
        return fail(TA_ERR_INVALID_ARG, "%s: bad o_dtype %d", fn, o_dtype);
    if (!std::isfinite(softmax_scale) || !(softmax_scale > 0.f))
        return fail(TA_ERR_INVALID_ARG, "%s: softmax_scale must be finite and > 0", fn);
    if (!std::isfinite(softcap) || softcap < 0.f)
        return fail(TA_ERR_INVALID_ARG, "%s: softcap must be finite and >= 0", fn);
    if (softcap > kRowsMaxCap)
        return fail(TA_ERR_UNSUPPORTED, "%s: softcap %g > %g", fn, softcap, kRowsMaxCap);
    if (softcap == 0.f && !slopes)
        return fail(TA_ERR_INVALID_ARG, "%s: neither a softcap nor slopes (plain scores are the "
                    "other passes')", fn);
    ScoredArgs a{};
    if (!rows_score_args(a.score, softmax_scale, softcap, slopes))
        return fail(TA_ERR_INVALID_ARG, "%s: softcap too small for the scale", fn);
    const int64_t base = kHdrWords + (int64_t)info->n_items * kItemWords +
                         (int64_t)info->n_merge_items * kMergeWords;
    const int64_t lists = info->kind == TA_KIND_BLOCKSPARSE ? info->window : 0;
    if (info->n_items < 0 || info->n_merge_items < 0 || info->n_partial_rows < 0 || lists < 0 ||
        info->words != base + lists)
        return fail(TA_ERR_SCHEDULE_MISMATCH, "%s: corrupt schedule info", fn);
    if (2LL * hq * head_dim >= (1LL << 24))
        return fail(TA_ERR_UNSUPPORTED, "%s: hq * head_dim too large", fn);
    const int64_t group = hq / hkv;
    // Eight waves, half of them in turns, share each K/V tile copied; four run two
    // workgroups to a CU (three at d = 64), which suits what the vector units
    // bound, finer launches and row blocks that do not come in eights.  Eight
    // where they pay: d = 128, whole eights of row blocks, and more than two
    // workgroups to a CU.  us with eight and with four waves: capped causal at d =
    // 128, 32 heads over 8, 700 tokens 28 and 21, 2500 tokens 79 and 74, 4000 tokens
    // (512 workgroups of eight) 150 and 163, 5500 tokens 285 and 282, 16384 tokens
    // 2205 and 2318; slopes, window 1024, 4000 tokens 94 and 94, packed 42000 tokens,
    // window 2048 1397 and 1504; 28 heads over 4, 8000 tokens 541 and 507; d = 64,
    // 12000 tokens 920 and 848.
    const int64_t blocks = group * (info->tile / 32);
    const bool eight = head_dim == 128 && blocks % 8 == 0 &&
                       info->n_items * (blocks / 8) * hkv > 512;
    const int nw = eight ? 8 : 4;
    const int64_t subtiles = (blocks + nw - 1) / nw;
    const int64_t wgs = info->n_items * subtiles * hkv;
    if (wgs * nw * 64 > UINT32_MAX)  // threads of a launch
        return fail(TA_ERR_UNSUPPORTED, "%s: grid too large", fn);
    if (info->n_items == 0)
        return TA_OK;
    if (!q || !k || !v || !o || !sched_dev)
        return fail(TA_ERR_INVALID_ARG, "%s: NULL q, k, v, o or schedule", fn);
    if (((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)o) & 15)
        return fail(TA_ERR_INVALID_ARG, "%s: q, k, v and o must be 16-byte aligned", fn);
    const size_t need = ta_workspace_bytes(info, hq, head_dim);
    if (need > 0 && (!workspace || workspace_bytes < need))
        return fail(TA_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, got %zu", fn, need,
                    workspace ? workspace_bytes : (size_t)0);
    if ((uintptr_t)workspace & 15)
        return fail(TA_ERR_INVALID_ARG, "%s: workspace must be 16-byte aligned", fn);
    a.q = static_cast<const uint16_t *>(q);
    a.k = static_cast<const uint16_t *>(k);
    a.v = static_cast<const uint16_t *>(v);
    a.o = o;
    a.lse = lse;
    a.sched = sched_dev;
    if (need > 0) {
        const size_t rows = (size_t)info->n_partial_rows * (size_t)hq;
        a.part_o = static_cast<float *>(workspace);
        a.part_lse = reinterpret_cast<float *>(
            static_cast<char *>(workspace) +
            ((rows * (size_t)head_dim * 4 + 255) & ~(size_t)255));
    }
    a.total_tokens = total_tokens;
    a.list_base = base;
    a.list_words = lists;
    a.kind = info->kind;
    a.tile = info->tile;
    a.hq = hq;
    a.hkv = hkv;
    a.group = (int32_t)group;
    a.sink = info->sink;
    a.window = info->window;
    a.n_items = info->n_items;
    a.n_merges = info->n_merge_items;
    a.n_partial_rows = need > 0 ? info->n_partial_rows : 0;
    a.subtiles = (int32_t)subtiles;
    a.o_f32 = o_dtype == TA_OUT_F32;
    const int score = (softcap > 0.f ? kScoreCap : 0) | (slopes ? kScoreSlope : 0);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const dim3 grid((uint32_t)wgs);
    const bool list = info->kind == TA_KIND_BLOCKSPARSE;
    if (head_dim == 128 && nw == 8)
        launch_scored<128, 8>(list, score, grid, s, a);
    else if (head_dim == 128)
        launch_scored<128, 4>(list, score, grid, s, a);
    else
        launch_scored<64, 4>(list, score, grid, s, a);
    hipError_t err = hipGetLastError();
    if (err == hipSuccess && a.n_merges > 0) {
        const dim3 join((uint32_t)((info->tile * hq + 3) / 4),
                        (uint32_t)std::min(a.n_merges, 65535));
        if (head_dim == 128)
            hipLaunchKernelGGL(scored_join_kernel<128>, join, dim3(kJoinThreads), 0, s, a);
        else
            hipLaunchKernelGGL(scored_join_kernel<64>, join, dim3(kJoinThreads), 0, s, a);
        err = hipGetLastError();
    }
    if (err != hipSuccess)
        return fail(TA_ERR_HIP, "%s: %s", fn, hipGetErrorString(err));
    return TA_OK;
}
