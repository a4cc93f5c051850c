// Attention over the paged K/V cache of libtriattn.so: single tokens, drafted
// tokens and pieces of prompts, with a prefix that the whole batch shares.
//
// Work.  The query rows of one kv head's group, (token, head of the group) in
// token-major order, are cut per request into row tiles of ROWS rows; the keys
// of a row tile into steps.  Laid end to end, the steps of all row tiles of a
// kv head are cut into equal shares, one a workgroup, so that the load is even
// whatever the lengths: a few long requests spread over the chip, many short
// ones share a workgroup.  Lengths are read on the device (a captured call
// follows them), each workgroup scanning the requests for itself.  A row tile
// whose steps fall into several shares leaves normalised fp32 partials and
// their log-sum-exp, joined in key order by a second kernel: results depend on
// the shape alone, not on timing.
//
// The shared prefix is one more such pass, in which the rows of all requests
// together attend to the prefix's keys: each K/V tile is read once for up to
// 128 rows instead of once a request; the join adds its partials to those of a
// row's own keys.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "triattn_device.h"
#include "triattn_internal.h"
#include "triattn_rows.h"
#include "triattn_spans.h"

namespace triattn {

int page_log2(int32_t page_size);  // triattn_cache.hip

namespace {

constexpr int kJoinThreads = 256;
constexpr int kMaxTiles = 2048;    // row tiles of a kv head
constexpr int kPageEntries = 512;  // page ids held in LDS at a time
constexpr int kCus = 256;

// What the own-keys pass leaves for the join, eight words a record: of every row
// tile where a prefix comes before, otherwise of each share the row tile that
// the share's start is the first to cut.  No rows: nothing to join.
constexpr int kRecordWords = 8;
enum RecordField { RF_Q0 = 0, RF_RHO0, RF_ROWS, RF_POS0, RF_BEGIN, RF_END, RF_SHARE };

struct PagedArgs {
    const uint16_t *q, *kc, *vc;
    void *o;
    float *lse;
    const int32_t *kv_lens, *cu_q, *table, *prefix_pages;
    float *slot_o, *slot_lse;  // pieces of row tiles: [2 slots, hkv, ROWS (, D)]
    float *row_o, *row_lse;    // whole row tiles that the join still needs: [T, hq (, D)]
    int32_t *records;
    ScoreArgs score;
    int32_t total_tokens, batch, width, hq, hkv, group;
    uint32_t group_inv;  // 65536 / group + 1: x * group_inv >> 16 = x / group, x < 2^13
    int32_t page_log2, num_pages, prefix_len;
    int32_t slots;      // shares a kv head
    int32_t max_tiles;  // row tiles that the call counts on at most
    int32_t n_records;
    int32_t o_f32;
};

// Shapes of the two forms of the pass.
//   RB = 1: up to 32 rows, bound by the bytes of K and V.  Two waves take 32-key
//     tiles in turn, each into two stages of its own, and keep their own softmax:
//     nothing waits on the other wave until they are joined at the end of a
//     piece.  64 KB of stages at d = 128 (32 KB at d = 64) let two workgroups
//     (four) share a CU, so that one loads while the other finds its next request
//     or joins its waves.  The tables of lengths come on top, 16 to 20 bytes a
//     request with query offsets and 8 without: fewer share a CU from some 700
//     requests with offsets on at d = 128, from 280 (700 without) at d = 64.
//   RB = 4: four waves of 32 rows each over the same 64-key tiles, in two stages.
template <int D, int RB>
struct PagedShape {
    static constexpr int NKB = RB == 4 ? 2 : 1;
    static constexpr int TK = 32 * NKB;      // keys of a tile
    static constexpr int KS = RB == 4 ? 1 : 2;  // key splits of a workgroup
    static constexpr int THREADS = 64 * RB * KS;
    static constexpr int STEP = TK * KS;     // keys of a step
    static constexpr int ROWS = 32 * RB;
    static constexpr int TILE_BYTES = TK * 2 * D;
    static constexpr int STAGE_BYTES = 2 * TILE_BYTES;  // K tile, then V tile
    static constexpr int LDS_BYTES = KS * 2 * STAGE_BYTES;
    // Least steps of a share: one of a 128-row tile leaves partials of twice
    // its K and V tiles' bytes.  us with 1, 4 and 8 steps (32 heads over 8, d =
    // 128): the last 64 tokens of 2000 27, 25, 29, of four times 1000 29, 25, 28,
    // 128 single tokens behind a prefix of 2048 47, 43, 44, the last 100 tokens of
    // 500 17, 24, 29; from 3000 keys on the same.
    static constexpr int LEAST = RB == 4 ? 4 : 1;
    static constexpr int WGS_PER_CU = RB == 1 && D == 64 ? 4 : 2;
    static constexpr int WAVES_PER_SIMD = (WGS_PER_CU * THREADS / 64 + 3) / 4;
};

// Exclusive scan of val(i), i < n, into out[0 .. n] (out[n]: the total) by
// the workgroup.
template <int kThreads, typename F>
__device__ __forceinline__ void block_scan(int n, int32_t *out, int32_t *wave_sum, F &&val)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int per = (n + kThreads - 1) / kThreads;
    int32_t sum = 0;
    for (int i = tid * per; i < min(n, (tid + 1) * per); ++i) {
        out[i] = sum;
        sum += val(i);
    }
    int32_t inc = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int32_t y = __shfl_up(inc, o);
        inc += lane >= o ? y : 0;
    }
    if (lane == 63)
        wave_sum[wave] = inc;
    __syncthreads();
    int32_t base = inc - sum, total = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) {
        base += w < wave ? wave_sum[w] : 0;
        total += wave_sum[w];
    }
    for (int i = tid * per; i < min(n, (tid + 1) * per); ++i)
        out[i] += base;
    if (tid == 0)
        out[n] = total;
    __syncthreads();
}

// The last i with start[i] <= x < start[i + 1], start ascending with
// start[0] <= x < start[n].
__device__ __forceinline__ int find_start(const int32_t *start, int n, int32_t x)
{
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (start[mid] <= x)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}

struct RowTile {
    int32_t q0;     // first token of the request
    int32_t rho0;   // first row of the tile in the request
    int32_t rows;   // rows of the tile
    int32_t pos0;   // position of the request's first query token
    int32_t limit;  // keys that some row of the tile keeps
    int32_t req;
    int32_t bad;    // a length past the block table
};

template <int D, int RB, int SCORE, bool PREFIX>
__global__ __launch_bounds__((PagedShape<D, RB>::THREADS),
                             (PagedShape<D, RB>::WAVES_PER_SIMD)) void paged_attn_kernel(PagedArgs a)
{
    using S = PagedShape<D, RB>;
    constexpr int kThreads = S::THREADS;
    constexpr int ROW_BYTES = 2 * D;
    constexpr int CHUNKS = D / 8;
    constexpr int COPY_ROWS = 1024 / ROW_BYTES;          // keys of a 1 KB copy
    constexpr int GROUP = 16;  // keys that surely share a page
    constexpr int COPIES = GROUP / COPY_ROWS;              // 1 KB copies of a group
    constexpr int GROUPS = S::TK / GROUP / (RB == 4 ? 4 : 1);  // of a wave and tile
    constexpr int D_BLOCKS = D / 32;

    __shared__ __attribute__((aligned(1024))) unsigned char smem[S::LDS_BYTES];
    // tables of the own-keys pass, as long as the call needs (table_bytes)
    extern __shared__ int32_t tables[];
    int32_t *const s_step = tables;                   // first step of a row tile, and the total
    int32_t *const s_kv = s_step + a.max_tiles + 1;   // own keys of a request
    int32_t *const s_req = s_kv + a.batch;            // first row tile of a request, and all
    int32_t *const s_cu = s_req + a.batch + 1;        // query offsets
    __shared__ int32_t s_page[kPageEntries];
    __shared__ int32_t s_wave[kThreads / 64];
    __shared__ float s_ml[S::KS][32][2];
    __shared__ int32_t s_bad;      // query offsets that are none
    __shared__ int32_t s_bad_key;  // first key of the piece in a page that is none

    const int tid = threadIdx.x;
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = blockIdx.x % a.hkv;
    const int slot = blockIdx.x / a.hkv;
    // a value that is the same on every lane, in a scalar register
    auto uni = [](int x) TA_INLINE -> int { return __builtin_amdgcn_readfirstlane(x); };
    auto div_group = [&](int x) TA_INLINE -> int {
        // row numbers pass 2^13 in prompts: a division there
        return x < 8192 ? (int)((uint32_t)x * a.group_inv >> 16) : x / a.group;
    };

    // The row tiles and where each one's steps begin.
    int n_tiles, total;
    const int32_t prefix_steps = PREFIX ? (a.prefix_len + S::STEP - 1) / S::STEP : 0;
    auto tile_of = [&](int t) TA_INLINE -> RowTile {
        RowTile r;
        r.bad = 0;
        if constexpr (PREFIX) {
            r.q0 = 0;
            r.rho0 = t * S::ROWS;
            r.rows = min(S::ROWS, a.total_tokens * a.group - r.rho0);
            r.pos0 = 0;
            r.limit = a.prefix_len;
            r.req = 0;
        } else {
            int nq = 1;
            r.req = t;
            r.q0 = t;
            r.rho0 = 0;
            if (a.cu_q) {
                r.req = find_start(s_req, a.batch, t);
                r.q0 = s_cu[r.req];
                nq = s_cu[r.req + 1] - r.q0;
                r.rho0 = (t - s_req[r.req]) * S::ROWS;
            }
            int32_t kv = s_kv[r.req];
            r.bad = kv > (a.width << a.page_log2);
            kv = r.bad ? 0 : max(kv, 0);
            r.rows = min(S::ROWS, nq * a.group - r.rho0);
            r.pos0 = kv - nq;
            r.limit = max(0, r.pos0 + div_group(r.rho0 + r.rows - 1) + 1);
        }
        return r;
    };
    if constexpr (PREFIX) {
        n_tiles = (a.total_tokens * a.group + S::ROWS - 1) / S::ROWS;
        total = n_tiles * prefix_steps;
    } else {
        n_tiles = a.batch;
        if (a.cu_q) {
            if (tid == 0)
                s_bad = 0;
            __syncthreads();
            bool bad = tid == 0 && (a.cu_q[0] != 0);
            block_scan<kThreads>(a.batch, s_req, s_wave, [&](int b) TA_INLINE -> int32_t {
                const int32_t b0 = a.cu_q[b], b1 = a.cu_q[b + 1];
                s_kv[b] = a.kv_lens[b];
                s_cu[b] = b0;
                if (b + 1 == a.batch)
                    s_cu[b + 1] = b1;
                if (b0 < 0 || b1 < b0 || b1 > a.total_tokens) {
                    bad = true;
                    return 0;
                }
                return ((b1 - b0) * a.group + S::ROWS - 1) / S::ROWS;
            });
            if (bad)
                s_bad = 1;
            __syncthreads();
            n_tiles = uni(s_req[a.batch]);
            // query offsets that are none: nothing is computed, NaN shows it
            if (s_bad != 0 || n_tiles > a.max_tiles) {
                if (g == 0)
                    for (int i = slot * kThreads + tid; i < a.n_records; i += a.slots * kThreads)
                        a.records[i * kRecordWords + RF_ROWS] = 0;
                poison_outputs(a.o, a.o_f32, a.lse, a.total_tokens, a.hq, D, blockIdx.x, gridDim.x);
                return;
            }
        }
        block_scan<kThreads>(n_tiles, s_step, s_wave, [&](int t) TA_INLINE -> int32_t {
            if (!a.cu_q)
                s_kv[t] = a.kv_lens[t];
            return (tile_of(t).limit + S::STEP - 1) / S::STEP;
        });
        total = uni(s_step[n_tiles]);
    }
    const int share = max(S::LEAST, (total + a.slots - 1) / a.slots);
    const int share0 = slot * share;
    const int share1 = min(total, share0 + share);
    if constexpr (!PREFIX) {
        // the records for the join
        auto record = [&](int i, int t) TA_INLINE {
            int32_t *m = a.records + kRecordWords * i;
            if (t < 0 || t >= n_tiles || s_step[t] == s_step[t + 1]) {
                m[RF_ROWS] = 0;
                return;
            }
            const RowTile r = tile_of(t);
            m[RF_Q0] = r.q0;
            m[RF_RHO0] = r.rho0;
            m[RF_ROWS] = r.rows;
            m[RF_POS0] = r.pos0;
            m[RF_BEGIN] = s_step[t];
            m[RF_END] = s_step[t + 1];
            m[RF_SHARE] = share;
        };
        if (g == 0 && a.row_o) {
            for (int i = slot * kThreads + tid; i < a.n_records; i += a.slots * kThreads)
                record(i, i);
        } else if (g == 0 && tid == 0) {
            int t = -1;
            if (share0 < total) {
                t = find_start(s_step, n_tiles, share0);
                if (s_step[t] == share0 || s_step[t] < share0 - share)
                    t = -1;  // not cut, or cut by an earlier share's start
            }
            record(slot, t);
        }
        // rows without keys, shared out over the slots
        for (int t = slot; t < n_tiles; t += a.slots) {
            if (s_step[t] != s_step[t + 1])
                continue;
            const RowTile r = tile_of(t);
            const float o = r.bad ? __builtin_nanf("") : 0.f;
            for (int i = tid; i < r.rows * D; i += kThreads) {
                const int rho = r.rho0 + i / D, qt = div_group(rho);
                const int h = g * a.group + rho - qt * a.group;
                const int64_t at = ((int64_t)(r.q0 + qt) * a.hq + h) * D + i % D;
                if (a.o_f32)
                    static_cast<float *>(a.o)[at] = o;
                else
                    static_cast<__bf16 *>(a.o)[at] = (__bf16)o;
                if (a.lse && i % D == 0)
                    a.lse[(int64_t)h * a.total_tokens + r.q0 + qt] = r.bad ? o : -INFINITY;
            }
        }
    }
    if (share0 >= total)
        return;

    const uint32_t smem_addr =
        (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)smem;
    // this wave's buffers (RB = 1) or the workgroup's stages (RB = 4)
    const int wave_lds = RB == 1 ? wave * 2 * S::STAGE_BYTES : 0;
    const int first_group = RB == 1 ? 0 : wave * GROUPS;
    const int dma_row = lane / CHUNKS;
    // a copying lane's place in a group's first block; block m flips the K
    // swizzle's bits of m COPY_ROWS
    const uint32_t dma_k =
        (uint32_t)(dma_row * ROW_BYTES + (((lane % CHUNKS) ^ rows_kswz<D>(dma_row)) << 4));
    const uint32_t dma_v =
        (uint32_t)(dma_row * ROW_BYTES + (((lane % CHUNKS) ^ rows_vswz<D>(dma_row)) << 4));
    const int64_t page_stride = ((int64_t)a.hkv << a.page_log2) * ROW_BYTES;
    const int64_t head_off = ((int64_t)g << a.page_log2) * ROW_BYTES;
    const unsigned char *kc = reinterpret_cast<const unsigned char *>(a.kc) + head_off;
    const unsigned char *vc = reinterpret_cast<const unsigned char *>(a.vc) + head_off;
    const int page_mask = (1 << a.page_log2) - 1;

    RowBlock<D, S::NKB, SCORE> rb;
    rb.init(lane);

    for (int at = share0, t = -1; at < share1;) {
        // the row tile of step `at`
        int t_begin, t_end;
        if constexpr (PREFIX) {
            t = at / prefix_steps;
            t_begin = t * prefix_steps;
            t_end = t_begin + prefix_steps;
        } else {
            if (t < 0)
                t = find_start(s_step, n_tiles, at);
            else
                do
                    ++t;
                while (s_step[t + 1] <= at);
            t = uni(t);
            t_begin = uni(s_step[t]);
            t_end = uni(s_step[t + 1]);
        }
        RowTile rt = tile_of(t);
        rt.q0 = uni(rt.q0);
        rt.rho0 = uni(rt.rho0);
        rt.rows = uni(rt.rows);
        rt.pos0 = uni(rt.pos0);
        rt.limit = uni(rt.limit);
        rt.req = uni(rt.req);
        const int step0 = at - t_begin;
        const int step1 = min(share1, t_end) - t_begin;
        const bool whole = step0 == 0 && step1 == t_end - t_begin;
        const int piece = 2 * slot + (t_begin > share0 ? 1 : 0);
        at = t_begin + step1;

        // this lane's query row (rows past the tile repeat its last one)
        const int block0 = RB == 1 ? 0 : 32 * wave;  // the wave's first row in the tile
        const int row = min(block0 + rb.col, rt.rows - 1);
        const int rho = rt.rho0 + row;
        const int tq = div_group(rho);
        const int head = g * a.group + rho - tq * a.group;
        const int tok = rt.q0 + tq;
        rb.load_q(a.q + ((int64_t)tok * a.hq + head) * D);
        float slope = 0.f;
        if constexpr ((SCORE & kScoreSlope) != 0)
            slope = a.score.slopes[head] * kRowsLog2e;
        // the last key that this row keeps, and the first row's: steps up to
        // that one need no mask
        const int last = PREFIX ? a.prefix_len - 1 : rt.pos0 + tq;
        const int first_last =
            PREFIX ? a.prefix_len - 1
                   : rt.pos0 + div_group(rt.rho0 + min(block0, rt.rows - 1));
        const int tile_first_last =
            PREFIX ? a.prefix_len - 1 : rt.pos0 + div_group(rt.rho0);
        // Where distances are taken from, so that they are short at the keys
        // that weigh most and round to little there: the row where scores fall
        // with the distance (in the prefix pass the prefix's end: the join adds
        // what each row is past it), the first key of all where they grow with
        // it (the log-sum-exp gets what the row is past that at its very end).
        int dist_row = PREFIX ? a.prefix_len : last;
        if constexpr ((SCORE & kScoreSlope) != 0)
            if (slope < 0.f)
                dist_row = PREFIX ? 0 : -a.prefix_len;
        const int32_t *pages = PREFIX ? a.prefix_pages : a.table + (int64_t)rt.req * a.width;
        if (tid == 0)
            s_bad_key = INT32_MAX;
        // One pass over the piece's steps.  Returns whether a masked step holds
        // infinite or NaN values; the `careful` pass then keeps them from the
        // rows that do not keep their keys.
        auto pass = [&](auto careful) TA_INLINE -> bool {
        constexpr bool CAREFUL = decltype(careful)::value;
        bool fresh = true, odd = false;
        rb.reset();
        const int seg_steps = (((kPageEntries - 1) << a.page_log2) / S::STEP);
        const int n_segs = (step1 - step0 + seg_steps - 1) / seg_steps;
        // where scores fall with the distance, the last keys come first: their
        // scores are the largest, and the rows' references stand
        constexpr bool BACK = (SCORE & kScoreSlope) != 0;
        for (int sg = 0; sg < n_segs; ++sg) {
            const int seg0 = step0 + (BACK ? n_segs - 1 - sg : sg) * seg_steps;
            const int seg1 = min(step1, seg0 + seg_steps);
            const int key_end = min(seg1 * S::STEP, rt.limit);
            const int page0 = (seg0 * S::STEP) >> a.page_log2;
            const int n_pages = ((key_end - 1) >> a.page_log2) + 1 - page0;
            __syncthreads();  // the last segment's ids, and buffers, are done with
            for (int i = tid; i < n_pages; i += kThreads) {
                int32_t id = pages[page0 + i];
                if (id < 0 || id >= a.num_pages) {
                    id = 0;
                    atomicMin(&s_bad_key, (page0 + i) << a.page_log2);
                }
                s_page[i] = id;
            }
            __syncthreads();

            // This wave's copies of a tile's K or V rows.  Keys from rt.limit on
            // repeat the last one before it; they lie past every row's last
            // key.
            auto copy = [&](int key0, uint32_t lds, auto is_v) TA_INLINE {
                constexpr bool V = decltype(is_v)::value;
                asm volatile("" ::: "memory");
                // lane i of the first GROUPS holds the page of this wave's group i
                const int mine =
                    min(key0 + (first_group + (lane & (GROUPS - 1))) * GROUP, rt.limit - 1);
                const int ids = s_page[(mine >> a.page_log2) - page0];
                const bool inside = key0 + S::TK <= rt.limit;
#pragma unroll
                for (int i = 0; i < GROUPS; ++i) {
                    const int gr = first_group + i;
                    const int key = key0 + gr * GROUP;
                    const unsigned char *page =
                        (V ? vc : kc) + (int64_t)__builtin_amdgcn_readlane(ids, i) * page_stride;
                    const uint32_t to = smem_addr + lds + gr * GROUP * ROW_BYTES;
                    uint32_t off[COPIES];
#pragma unroll
                    for (int m = 0; m < COPIES; ++m)
                        off[m] = V ? dma_v : dma_k ^ (uint32_t)(rows_kswz<D>(m * COPY_ROWS) << 4);
                    if (inside) {
                        copy_burst_to_lds16<COPIES>(page + (key & page_mask) * ROW_BYTES, off, to);
                    } else {
#pragma unroll
                        for (int m = 0; m < COPIES; ++m) {
                            const int first = min(key + m * COPY_ROWS, rt.limit - 1);
                            const int lim = rt.limit - 1 - first;  // rows after the first
                            copy_to_lds16(page + (first & page_mask) * ROW_BYTES,
                                          off[m] - (uint32_t)(max(dma_row - lim, 0) * ROW_BYTES),
                                          to + m * 1024);
                        }
                    }
                }
                asm volatile("" ::: "memory");
            };
            using K = std::false_type;
            using V = std::true_type;
            f32x16 s[S::NKB];
            bf16x8 p[S::NKB][2];
            auto softmax = [&](int key0) TA_INLINE {
                rb.modify(s, a.score);
                if (__builtin_expect(key0 + S::TK - 1 > first_last, 0)) {
                    asm volatile("");  // a branch: most steps have no mask
                    rb.mask_above(s, last - key0);
                }
                rb.softmax(s, a.score, slope, key0 - dist_row, p, fresh);
                fresh = false;
            };
            auto values = [&](int key0, const unsigned char *vt) TA_INLINE {
                // (a step that any of the tile's rows masks: the waves look at a
                // part of the values each)
                if (__builtin_expect(key0 + S::TK - 1 > tile_first_last, 0)) {
                    asm volatile("");
                    odd |= rb.odd_values(vt, lane, RB == 1 ? 0 : wave, RB);
                }
                __builtin_amdgcn_sched_barrier(0);
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
            if constexpr (CAREFUL) {
                // tile by tile, in this wave's first stage (RB = 1) or the
                // workgroup's
                const int n = (key_end - seg0 * S::STEP + S::STEP - 1) / S::STEP;
                for (int i = 0; i < n; ++i) {
                    const int key0 = (seg0 + (BACK ? n - 1 - i : i)) * S::STEP +
                                     (RB == 1 ? wave * S::TK : 0);
                    const bool on = key0 < key_end;
                    if (on) {
                        copy(key0, wave_lds, K{});
                        copy(key0, wave_lds + S::TILE_BYTES, V{});
                    }
                    rows_wait_copies<0>();
                    barrier_no_fence();
                    if (on) {
                        products(smem + wave_lds);
                        softmax(key0);
                        rb.accumulate_by_key(smem + wave_lds + S::TILE_BYTES, s, p);
                    }
                    barrier_no_fence();
                }
            } else if constexpr (RB == 1) {
                // tiles of this wave: key0 = step STEP + wave TK
                const int base = seg0 * S::STEP + wave * S::TK;
                const int n = base < key_end ? (key_end - base + S::STEP - 1) / S::STEP : 0;
                auto key_of = [&](int i) TA_INLINE -> int {
                    return base + (BACK ? n - 1 - i : i) * S::STEP;
                };
                auto copies = [&](int key0, int stage) TA_INLINE {
                    copy(key0, wave_lds + stage * S::STAGE_BYTES, K{});
                    copy(key0, wave_lds + stage * S::STAGE_BYTES + S::TILE_BYTES, V{});
                    __builtin_amdgcn_sched_barrier(0);
                };
                if (n > 0)
                    copies(key_of(0), 0);
                if (n > 1)
                    copies(key_of(1), 1);
                auto step = [&](int i, auto stage) TA_INLINE {
                    constexpr int ST = decltype(stage)::value;
                    const unsigned char *kt = smem + wave_lds + ST * S::STAGE_BYTES;
                    if (i + 1 < n)
                        rows_wait_copies<2 * GROUPS * COPIES>();
                    else
                        rows_wait_copies<0>();
                    products(kt);
                    softmax(key_of(i));
                    values(key_of(i), kt + S::TILE_BYTES);
                    if (i + 2 < n) {
                        // every read of the stage has returned before it is
                        // written again
                        __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
                        copies(key_of(i + 2), ST);
                    }
                };
                int i = 0;
                for (; i + 1 < n; i += 2) {
                    step(i, std::integral_constant<int, 0>{});
                    step(i + 1, std::integral_constant<int, 1>{});
                }
                if (i < n)
                    step(i, std::integral_constant<int, 0>{});
            } else {
                const int n = (key_end - seg0 * S::STEP + S::STEP - 1) / S::STEP;
                // Where step i's keys are: wave w copies the tile's w-th group.
                // Found a step ahead, so that the copies go out between the first
                // matrix instructions of a step without waiting for page ids.
                struct Place {
                    int key0;
                    uint32_t lim;  // byte offset of the group's last row
                    int64_t off;   // bytes to its first row
                };
                auto place = [&](int i) TA_INLINE -> Place {
                    Place x;
                    x.key0 = (seg0 + (BACK ? n - 1 - i : i)) * S::STEP;
                    const int first = min(x.key0 + wave * GROUP, rt.limit - 1);
                    x.lim = (uint32_t)(min(rt.limit - 1 - first, GROUP - 1) * ROW_BYTES);
                    const int id = uni(s_page[(first >> a.page_log2) - page0]);
                    x.off = (int64_t)id * page_stride + (first & page_mask) * ROW_BYTES;
                    return x;
                };
                const uint32_t row_off = (uint32_t)(dma_row * ROW_BYTES);
                auto copy_block = [&](const Place &x, int c, int stage) TA_INLINE {
                    const bool v = c >= COPIES;
                    const int m = v ? c - COPIES : c;
                    const uint32_t swz =
                        v ? dma_v - row_off
                          : (dma_k - row_off) ^ (uint32_t)(rows_kswz<D>(m * COPY_ROWS) << 4);
                    copy_to_lds16((v ? vc : kc) + x.off,
                                  min(row_off + (uint32_t)(m * 1024), x.lim) + swz,
                                  smem_addr + stage * S::STAGE_BYTES + (v ? S::TILE_BYTES : 0) +
                                      wave * GROUP * ROW_BYTES + m * 1024);
                };
                constexpr int STRIDE = S::NKB * (D / 16) / (2 * COPIES);
                Place now = place(0), next = place(min(1, n - 1));
#pragma unroll
                for (int c = 0; c < 2 * COPIES; ++c)
                    copy_block(now, c, 0);
                auto step = [&](int i, auto stage) TA_INLINE {
                    constexpr int ST = decltype(stage)::value;
                    // this step's tile has landed for every wave, and every
                    // wave is done with the other stage
                    __builtin_amdgcn_sched_barrier(0);
                    rows_wait_copies<0>();
                    barrier_no_fence();
                    __builtin_amdgcn_sched_barrier(0);
                    // (after the last step the copies repeat its tile, into the
                    // stage that nothing reads any more)
                    const unsigned char *kt = smem + ST * S::STAGE_BYTES;
                    rb.products(kt, s, [&](int m) TA_INLINE {
                        if (m % STRIDE == STRIDE - 1 && m / STRIDE < 2 * COPIES)
                            copy_block(next, m / STRIDE, 1 - ST);
                    });
                    rb.template schedule<true, false>();
                    __builtin_amdgcn_sched_barrier(0);
                    const int key0 = now.key0;
                    now = next;
                    next = place(min(i + 2, n - 1));
                    softmax(key0);
                    values(key0, kt + S::TILE_BYTES);
                };
                int i = 0;
                for (; i + 1 < n; i += 2) {
                    step(i, std::integral_constant<int, 0>{});
                    step(i + 1, std::integral_constant<int, 1>{});
                }
                if (i < n)
                    step(i, std::integral_constant<int, 0>{});
                rows_wait_copies<0>();
            }
        }
        return odd;
        };
        if (__builtin_expect(__syncthreads_or(pass(std::false_type{})), 0))
            pass(std::true_type{});

        // Where the rows go.
        const bool to_o = whole && !a.row_o;
        auto store4 = [&](f32x4r x, int r, int d0) TA_INLINE {
            const int rr = rt.rho0 + r, qt = div_group(rr);
            const int64_t orow =
                (int64_t)(rt.q0 + qt) * a.hq + g * a.group + rr - qt * a.group;
            if (to_o && !a.o_f32)
                *reinterpret_cast<bf16x4r *>(static_cast<__bf16 *>(a.o) + orow * D + d0) =
                    __builtin_convertvector(x, bf16x4r);
            else if (to_o)
                *reinterpret_cast<f32x4r *>(static_cast<float *>(a.o) + orow * D + d0) = x;
            else if (whole)
                *reinterpret_cast<f32x4r *>(a.row_o + orow * D + d0) = x;
            else
                *reinterpret_cast<f32x4r *>(
                    a.slot_o + (((int64_t)piece * a.hkv + g) * S::ROWS + r) * D + d0) = x;
        };
        auto store_lse = [&](float x, int r) TA_INLINE {
            const int rr = rt.rho0 + r, qt = div_group(rr);
            const int h = g * a.group + rr - qt * a.group;
            if (to_o) {
                if constexpr ((SCORE & kScoreSlope) != 0)
                    x += rows_lse_shift(a.score.slopes[h], rt.pos0 + qt);
                if (a.lse)
                    a.lse[(int64_t)h * a.total_tokens + rt.q0 + qt] = x;
            } else if (whole) {
                a.row_lse[(int64_t)(rt.q0 + qt) * a.hq + h] = x;
            } else {
                a.slot_lse[((int64_t)piece * a.hkv + g) * S::ROWS + r] = x;
            }
        };
        __syncthreads();  // the stages are done with, and s_bad_key is final
        // what a row whose last key is this one shows: NaN from the first page
        // that is none on (earlier rows of the tile do not keep its keys)
        const int bad_key = s_bad_key;
        auto nan_if_bad = [&](int last_key) TA_INLINE -> float {
            return last_key >= bad_key ? __builtin_nanf("") : 0.f;
        };
        if constexpr (RB == 1) {
            // join the waves: each leaves its accumulators in its buffers,
            // 16-byte chunks of row r permuted by r against bank conflicts
            constexpr int PITCH = 4 * D;
            static_assert(32 * PITCH <= 2 * S::STAGE_BYTES, "accumulators fit the wave's stages");
            auto place = [&](int r, int chunk) TA_INLINE -> int {
                return r * PITCH + ((chunk ^ (r & (D / 4 - 1))) << 4);
            };
            unsigned char *mine = smem + wave * 2 * S::STAGE_BYTES;
            const float l = rows_pair_sum(rb.l_run);
            if (rb.col < rt.rows) {
                if (rb.half == 0) {
                    s_ml[wave][rb.col][0] = rb.m_ref;
                    s_ml[wave][rb.col][1] = l;
                }
#pragma unroll
                for (int b = 0; b < D_BLOCKS; ++b)
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        f32x4r x;
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            x[e] = rb.oacc[b][4 * c + e];
                        *reinterpret_cast<f32x4r *>(
                            mine + place(rb.col, 8 * b + 2 * c + rb.half)) = x;
                    }
            }
            __syncthreads();
            for (int i = tid; i < rt.rows * (D / 4); i += kThreads) {
                const int r = i / (D / 4), d0 = 4 * (i % (D / 4));
                float m = -INFINITY;
#pragma unroll
                for (int w = 0; w < S::KS; ++w)
                    m = fmaxf(m, s_ml[w][r][0]);
                const float m_use = m == -INFINITY ? 0.f : m;
                float den = 0.f;
                f32x4r x{};
#pragma unroll
                for (int w = 0; w < S::KS; ++w) {
                    const float f = __builtin_amdgcn_exp2f(s_ml[w][r][0] - m_use);
                    den += f * s_ml[w][r][1];
                    const f32x4r y = *reinterpret_cast<const f32x4r *>(
                        smem + w * 2 * S::STAGE_BYTES + place(r, d0 / 4));
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        x[e] += f * y[e];
                }
                const float nan = nan_if_bad(PREFIX ? last : rt.pos0 + div_group(rt.rho0 + r));
                const float inv = (den == 0.f ? 0.f : 1.f / den) + nan;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    x[e] *= inv;
                store4(x, r, d0);
                if (d0 == 0)
                    store_lse((den == 0.f ? -INFINITY : (m + __log2f(den)) * kRowsLn2) + nan,
                              r);
            }
        } else if (block0 + rb.col < rt.rows) {
            float inv, lse;
            rb.finish(inv, lse);
            const float nan = nan_if_bad(last);
            inv += nan;
            lse += nan;
#pragma unroll
            for (int b = 0; b < D_BLOCKS; ++b)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    f32x4r x;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        x[e] = rb.oacc[b][4 * c + e] * inv;
                    store4(x, block0 + rb.col, 32 * b + 8 * c + 4 * rb.half);
                }
            if (rb.half == 0)
                store_lse(lse, block0 + rb.col);
        }
        __syncthreads();  // s_bad_key and the accumulators are read
    }
}

struct JoinArgs {
    void *o;
    float *lse;
    const int32_t *records;
    const float *slot_o, *slot_lse;
    int32_t tile_rows;
    int32_t chunks, chunk_rows;  // workgroups of a row tile, rows of each
    // the prefix pass (prefix_len 0: none)
    const float *row_o, *row_lse;
    const float *pre_slot_o, *pre_slot_lse, *pre_row_o, *pre_row_lse;
    int32_t prefix_len, pre_rows, pre_steps, pre_share;
    const float *slopes;
    int32_t total_tokens, hq, hkv, group, o_f32;
};

// Joins the partials of a row: O = sum_c w_c O_c / sum_c w_c with w_c =
// exp(LSE_c - max_c LSE_c), the prefix's before the row's own, in key order.
// With a prefix every row has partials to join; without one only the row tiles
// that a share's start cuts, which the shares name.  Sixteen lanes take a row:
// what bounds this is the chain of loads (cut, record, log-sum-exps, partials), so
// many rows at once matter more than wide ones (prompt pieces: 22 us, with a wave
// to a row 50).
template <int D>
__global__ __launch_bounds__(kJoinThreads) void paged_join_kernel(JoinArgs a)
{
    constexpr int LANES = 16;        // of a row
    constexpr int PER = D / LANES;   // values of a lane, in runs of four
    constexpr int RUNS = PER / 4;
    const int g = blockIdx.x % a.hkv, at = blockIdx.x / a.hkv;
    const int chunk = at % a.chunks;
    const int32_t *m = a.records + kRecordWords * (at / a.chunks);
    const int32_t q0 = m[RF_Q0], rho0 = m[RF_RHO0], rows = m[RF_ROWS], pos0 = m[RF_POS0];
    const int32_t begin = m[RF_BEGIN], end = m[RF_END], share = m[RF_SHARE];
    if (rows == 0)
        return;
    const int w0 = begin / share;
    const int n_own = (end - 1) / share - w0 + 1;
    const int lane = threadIdx.x % LANES;
    {
        const int r = chunk * a.chunk_rows + threadIdx.x / LANES;
        if (threadIdx.x / LANES >= a.chunk_rows || r >= rows)
            return;
        const int rho = rho0 + r, qt = rho / a.group, h = g * a.group + rho - qt * a.group;
        const int64_t orow = (int64_t)(q0 + qt) * a.hq + h;
        // the prefix pass's pieces of this row: its rows are those of all
        // requests, in the same order
        int n_pre = 0, pw0 = 0, prow = 0, pbegin = 0;
        float shift = 0.f;
        if (a.prefix_len > 0 && pos0 + qt >= 0) {
            const int prho = (q0 + qt) * a.group + rho - qt * a.group;
            pbegin = prho / a.pre_rows * a.pre_steps;
            prow = prho % a.pre_rows;
            pw0 = pbegin / a.pre_share;
            n_pre = (pbegin + a.pre_steps - 1) / a.pre_share - pw0 + 1;
            if (a.slopes && a.slopes[h] > 0.f)  // its distances end at the prefix's end
                shift = -a.slopes[h] * (float)(pos0 + qt);
        }
        const int n = n_pre + n_own;
        // row of partial c: in the whole rows or the pieces of its pass
        auto index = [&](int c) TA_INLINE -> int64_t {
            if (c < n_pre) {
                const int w = pw0 + c;
                return n_pre == 1 ? orow
                                  : ((int64_t)(2 * w + (pbegin > w * a.pre_share)) * a.hkv + g) *
                                            a.pre_rows + prow;
            }
            const int w = w0 + c - n_pre;
            return n_own == 1 ? orow
                              : ((int64_t)(2 * w + (begin > w * share)) * a.hkv + g) *
                                        a.tile_rows + r;
        };
        auto lse_of = [&](int c) TA_INLINE -> float {
            const float *from = c < n_pre ? (n_pre == 1 ? a.pre_row_lse : a.pre_slot_lse)
                                          : (n_own == 1 ? a.row_lse : a.slot_lse);
            return from[index(c)] + (c < n_pre ? shift : 0.f);
        };
        float mx = -INFINITY;
        for (int c = lane; c < n; c += LANES)
            mx = fmaxf(mx, lse_of(c));
#pragma unroll
        for (int o = LANES / 2; o >= 1; o >>= 1)
            mx = fmaxf(mx, __shfl_xor(mx, o));
        const float m_use = mx == -INFINITY ? 0.f : mx;
        f32x4r acc[RUNS] = {};
        float den = 0.f;
        for (int c0 = 0; c0 < n; c0 += LANES) {
            const float w = c0 + lane < n ? __expf(lse_of(c0 + lane) - m_use) : 0.f;
            den += w;  // (NaN stays visible)
            const int top = min(n - c0, LANES);
            constexpr int UNROLL = 8;
            for (int c = 0; c < top; c += UNROLL) {
                f32x4r x[UNROLL][RUNS];
#pragma unroll
                for (int u = 0; u < UNROLL; ++u) {
                    const int cc = c0 + min(c + u, top - 1);
                    const float *from = cc < n_pre ? (n_pre == 1 ? a.pre_row_o : a.pre_slot_o)
                                                   : (n_own == 1 ? a.row_o : a.slot_o);
                    from += index(cc) * D + 4 * lane;
#pragma unroll
                    for (int i = 0; i < RUNS; ++i)
                        x[u][i] = *reinterpret_cast<const f32x4r *>(from + 4 * LANES * i);
                }
#pragma unroll
                for (int u = 0; u < UNROLL; ++u) {
                    const float f = __shfl(w, min(c + u, top - 1), LANES);
                    if (c + u < top)
#pragma unroll
                        for (int i = 0; i < RUNS; ++i)
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                acc[i][e] += f * x[u][i][e];
                }
            }
        }
#pragma unroll
        for (int o = LANES / 2; o >= 1; o >>= 1)
            den += __shfl_xor(den, o);
        const float inv = den == 0.f ? 0.f : 1.f / den;
#pragma unroll
        for (int i = 0; i < RUNS; ++i) {
            const int64_t to = orow * D + 4 * LANES * i + 4 * lane;
            const f32x4r y = acc[i] * inv;
            if (a.o_f32)
                *reinterpret_cast<f32x4r *>(static_cast<float *>(a.o) + to) = y;
            else
                *reinterpret_cast<bf16x4r *>(static_cast<__bf16 *>(a.o) + to) =
                    __builtin_convertvector(y, bf16x4r);
        }
        if (a.lse && lane == 0)
            a.lse[(int64_t)h * a.total_tokens + q0 + qt] =
                den == 0.f ? -INFINITY
                           : m_use + __logf(den) +
                                 (a.slopes ? rows_lse_shift(a.slopes[h], a.prefix_len + pos0 + qt)
                                           : 0.f);
    }
}

// How a call is laid out: forms, shares and the parts of the workspace.
struct PagedLayout {
    int own_rb, pre_rb;        // row blocks of the two passes
    int own_slots, pre_slots;  // shares a kv head
    int max_tiles, n_records;
    size_t records, own_slot_o, own_slot_lse, own_row_o, own_row_lse, pre_slot_o, pre_slot_lse,
        pre_row_o, pre_row_lse, bytes;
};

int wgs_per_cu(int rb, int d)
{
    if (d == 128)
        return rb == 4 ? PagedShape<128, 4>::WGS_PER_CU : PagedShape<128, 1>::WGS_PER_CU;
    return rb == 4 ? PagedShape<64, 4>::WGS_PER_CU : PagedShape<64, 1>::WGS_PER_CU;
}

PagedLayout paged_layout(int32_t batch, int64_t total_tokens, bool ragged, bool prefix, int32_t hq,
                         int32_t hkv, int32_t d)
{
    PagedLayout p{};
    const int64_t group = hq / hkv;
    // Up to 32 rows a request on average: tiles of 32 rows, which a
    // workgroup's two waves share out by keys; 128 otherwise.  us with 32 and with
    // 128 (32 heads over 8, d = 128, 4000 keys a request): 64 requests of one
    // token 183 and 193, 24 of eight (32 rows) 93 and 96, of nine 133 and 97, of 32
    // 232 and 113.  One form serves the whole call, also where requests differ:
    // 64 single tokens and one piece of 400 (behind 8000 keys) 279 (as chosen) and
    // 242, one of 700 349 and 281 (as chosen; 184 and 113 in calls of their own);
    // 255 single tokens and one piece of 1024 915 (as chosen) and 823.
    p.own_rb = !ragged || total_tokens * group <= (int64_t)batch * 32 ? 1 : 4;
    p.pre_rb = total_tokens * group <= 32 ? 1 : 4;
    p.own_slots = std::max(1, kCus * wgs_per_cu(p.own_rb, d) / hkv);
    p.pre_slots = std::max(1, kCus * wgs_per_cu(p.pre_rb, d) / hkv);
    const int64_t rows = 32 * p.own_rb;
    p.max_tiles = (int)std::min<int64_t>(
        kMaxTiles + 1, ragged ? total_tokens * group / rows + batch : (int64_t)batch);
    size_t at = 0;
    auto take = [&](size_t n) {
        const size_t here = at;
        at += (n + 255) / 256 * 256;
        return here;
    };
    p.n_records = prefix ? p.max_tiles : p.own_slots;
    p.records = take((size_t)p.n_records * kRecordWords * 4);
    const size_t own = (size_t)2 * p.own_slots * hkv * rows;
    p.own_slot_o = take(own * d * 4);
    p.own_slot_lse = take(own * 4);
    if (prefix) {
        const size_t all = (size_t)total_tokens * hq;
        const size_t pre = (size_t)2 * p.pre_slots * hkv * 32 * p.pre_rb;
        p.own_row_o = take(all * d * 4);
        p.own_row_lse = take(all * 4);
        p.pre_slot_o = take(pre * d * 4);
        p.pre_slot_lse = take(pre * 4);
        p.pre_row_o = take(all * d * 4);
        p.pre_row_lse = take(all * 4);
    }
    p.bytes = at;
    return p;
}

// LDS of the own-keys pass's tables.
uint32_t table_bytes(const PagedArgs &a)
{
    return 4u * (uint32_t)(a.max_tiles + 1 + a.batch +
                           (a.cu_q ? 2 * (a.batch + 1) : 0));
}

template <int D, int RB, bool PREFIX>
void launch_scores(int score, dim3 grid, hipStream_t s, const PagedArgs &a)
{
    const dim3 threads(PagedShape<D, RB>::THREADS);
    const uint32_t lds = PREFIX ? 0 : table_bytes(a);
    switch (score) {
    case 0: hipLaunchKernelGGL((paged_attn_kernel<D, RB, 0, PREFIX>), grid, threads, lds, s, a); break;
    case 1: hipLaunchKernelGGL((paged_attn_kernel<D, RB, 1, PREFIX>), grid, threads, lds, s, a); break;
    case 2: hipLaunchKernelGGL((paged_attn_kernel<D, RB, 2, PREFIX>), grid, threads, lds, s, a); break;
    default: hipLaunchKernelGGL((paged_attn_kernel<D, RB, 3, PREFIX>), grid, threads, lds, s, a); break;
    }
}

template <bool PREFIX>
hipError_t launch_pass(int d, int rb, int score, hipStream_t s, const PagedArgs &a)
{
    const dim3 grid((uint32_t)(a.slots * a.hkv));
    if (d == 128 && rb == 1)
        launch_scores<128, 1, PREFIX>(score, grid, s, a);
    else if (d == 128)
        launch_scores<128, 4, PREFIX>(score, grid, s, a);
    else if (rb == 1)
        launch_scores<64, 1, PREFIX>(score, grid, s, a);
    else
        launch_scores<64, 4, PREFIX>(score, grid, s, a);
    return hipGetLastError();
}

}  // namespace
}  // namespace triattn

using namespace triattn;

extern "C" size_t ta_paged_workspace_bytes(int32_t batch, int64_t total_tokens, int32_t ragged,
                                           int32_t prefix, int32_t hq, int32_t hkv,
                                           int32_t head_dim)
{
    if (batch < 0 || total_tokens < 0 || total_tokens > INT32_MAX || hq <= 0 || hkv <= 0 ||
        hq % hkv != 0 || hq / hkv > 8 || (head_dim != 64 && head_dim != 128))
        return 0;
    return paged_layout(batch, total_tokens, ragged != 0, prefix != 0, hq, hkv, head_dim).bytes;
}

extern "C" ta_status paged_attn_fwd(const void *q, const void *k_cache, const void *v_cache,
                                    void *o, int32_t o_dtype, float *lse, const int32_t *kv_lens,
                                    const int32_t *cu_q, const int32_t *block_table, int32_t batch,
                                    int32_t table_width, const int32_t *prefix_pages,
                                    int32_t prefix_len, int64_t total_tokens, int32_t hq,
                                    int32_t hkv, int32_t head_dim, int64_t num_pages,
                                    int32_t page_size, float softmax_scale, float softcap,
                                    const float *slopes, void *workspace, size_t workspace_bytes,
                                    void *stream)
{
    clear_error();
    const char *fn = "paged_attn_fwd";
    if (batch < 0 || total_tokens < 0 || table_width < 0 || prefix_len < 0 || num_pages < 0)
        return fail(TA_ERR_INVALID_ARG, "%s: negative size", fn);
    if (hq <= 0 || hkv <= 0)
        return fail(TA_ERR_INVALID_ARG, "%s: hq and hkv must be positive", fn);
    if (hq % hkv != 0)
        return fail(TA_ERR_INVALID_ARG, "%s: hq %d not a multiple of hkv %d", fn, hq, hkv);
    if (hq / hkv > 8)
        return fail(TA_ERR_UNSUPPORTED, "%s: GQA group %d > 8", fn, hq / hkv);
    if (head_dim != 64 && head_dim != 128)
        return fail(TA_ERR_UNSUPPORTED, "%s: head_dim %d not in {64, 128}", fn, head_dim);
    const int lp = page_log2(page_size);
    if (lp < 0)
        return fail(TA_ERR_UNSUPPORTED, "%s: page_size %d not in {16, 32, 64, 128, 256}", fn,
                    page_size);
    if (o_dtype != TA_OUT_BF16 && o_dtype != TA_OUT_F32)
        return fail(TA_ERR_INVALID_ARG, "%s: bad o_dtype %d", fn, o_dtype);
    if (!std::isfinite(softmax_scale) || !(softmax_scale > 0.f))
        return fail(TA_ERR_INVALID_ARG, "%s: softmax_scale must be finite and > 0", fn);
    if (!std::isfinite(softcap) || softcap < 0.f)
        return fail(TA_ERR_INVALID_ARG, "%s: softcap must be finite and >= 0", fn);
    if (softcap > kRowsMaxCap)
        return fail(TA_ERR_UNSUPPORTED, "%s: softcap %g > %g", fn, softcap, kRowsMaxCap);
    ScoreArgs score_args;
    if (!rows_score_args(score_args, softmax_scale, softcap, slopes))
        return fail(TA_ERR_INVALID_ARG, "%s: softcap too small for the scale", fn);
    if (!cu_q && total_tokens != batch)
        return fail(TA_ERR_INVALID_ARG, "%s: %lld tokens for %d requests of one each", fn,
                    (long long)total_tokens, batch);
    if (batch > TA_MAX_BATCH)
        return fail(TA_ERR_UNSUPPORTED, "%s: batch %d > %d", fn, batch, TA_MAX_BATCH);
    // (keys are walked in whole steps, whose ends stay in 32 bits too)
    if (num_pages > INT32_MAX / page_size ||
        (int64_t)table_width * page_size > INT32_MAX - 256 || prefix_len > INT32_MAX - 256 ||
        (slopes && (int64_t)table_width * page_size + prefix_len > INT32_MAX - 256) ||
        (int64_t)total_tokens * hq > INT32_MAX)
        return fail(TA_ERR_UNSUPPORTED, "%s: positions, slots or rows past 32 bits", fn);
    const PagedLayout p =
        paged_layout(batch, total_tokens, cu_q != nullptr, prefix_len > 0, hq, hkv, head_dim);
    const int64_t group = hq / hkv;
    if (p.max_tiles > kMaxTiles)
        return fail(TA_ERR_UNSUPPORTED, "%s: more than %d row tiles a kv head (pass fewer query "
                    "tokens at a time)", fn, kMaxTiles);
    // steps are counted in 32 bits
    const int64_t steps = (int64_t)p.max_tiles * ((int64_t)table_width * page_size / 64 + 1);
    const int64_t pre_tiles = (total_tokens * group + 32 * p.pre_rb - 1) / (32 * p.pre_rb);
    if (steps > INT32_MAX / 2 || pre_tiles * (prefix_len / 64 + 1) > INT32_MAX / 2)
        return fail(TA_ERR_UNSUPPORTED, "%s: too many steps", fn);
    // the join: workgroups of a row tile, rows of each
    const int join_rows = cu_q ? 32 * p.own_rb : (int)group;
    const int chunk_rows = std::min(join_rows, kJoinThreads / 16);
    const int chunks = (join_rows + chunk_rows - 1) / chunk_rows;
    const int64_t wgs = std::max<int64_t>({p.own_slots, prefix_len > 0 ? p.pre_slots : 0,
                                           (int64_t)p.n_records * chunks}) * hkv;
    if (wgs * kJoinThreads > UINT32_MAX)  // threads of a launch
        return fail(TA_ERR_UNSUPPORTED, "%s: grid too large", fn);
    if (total_tokens == 0 || batch == 0)
        return TA_OK;
    if (!q || !o || !kv_lens || (num_pages > 0 && (!k_cache || !v_cache)) ||
        (table_width > 0 && !block_table) || (prefix_len > 0 && !prefix_pages))
        return fail(TA_ERR_INVALID_ARG, "%s: NULL argument", fn);
    if (num_pages == 0)
        return fail(TA_ERR_INVALID_ARG, "%s: a cache without pages", fn);
    if (((uintptr_t)q | (uintptr_t)k_cache | (uintptr_t)v_cache | (uintptr_t)o) & 15)
        return fail(TA_ERR_INVALID_ARG, "%s: q, o and the caches must be 16-byte aligned", fn);
    if (!workspace || workspace_bytes < p.bytes)
        return fail(TA_ERR_WORKSPACE, "%s: workspace of %zu bytes, need %zu", fn,
                    workspace ? workspace_bytes : (size_t)0, p.bytes);
    if ((uintptr_t)workspace & 15)
        return fail(TA_ERR_WORKSPACE, "%s: workspace must be 16-byte aligned", fn);
    {
        const int64_t rows = total_tokens * hq, cache = ((num_pages * hkv) << lp) * head_dim * 2;
        const Span spans[] = {{o, rows * head_dim * (o_dtype == TA_OUT_F32 ? 4 : 2)},
                              {lse, 4 * rows},
                              {workspace, (int64_t)p.bytes},
                              {q, rows * head_dim * 2},
                              {k_cache, cache},
                              {v_cache, cache},
                              {kv_lens, 4LL * batch},
                              {cu_q, 4LL * batch + 4},
                              {block_table, 4LL * batch * table_width},
                              {prefix_len > 0 ? prefix_pages : nullptr,
                               4 * (((int64_t)prefix_len + page_size - 1) >> lp)},
                              {slopes, 4LL * hq}};
        if (spans_overlap(spans, 3, 11))
            return fail(TA_ERR_INVALID_ARG, "%s: an output overlaps another argument", fn);
    }
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    auto part = [&](size_t off) { return reinterpret_cast<float *>(ws + off); };
    PagedArgs a{};
    a.q = static_cast<const uint16_t *>(q);
    a.kc = static_cast<const uint16_t *>(k_cache);
    a.vc = static_cast<const uint16_t *>(v_cache);
    a.o = o;
    a.lse = lse;
    a.kv_lens = kv_lens;
    a.cu_q = cu_q;
    a.table = block_table;
    a.prefix_pages = prefix_pages;
    a.slot_o = part(p.own_slot_o);
    a.slot_lse = part(p.own_slot_lse);
    const bool prefix = prefix_len > 0;
    a.row_o = prefix ? part(p.own_row_o) : nullptr;
    a.row_lse = prefix ? part(p.own_row_lse) : nullptr;
    a.records = reinterpret_cast<int32_t *>(ws + p.records);
    a.n_records = p.n_records;
    a.score = score_args;
    a.total_tokens = (int32_t)total_tokens;
    a.batch = batch;
    a.width = table_width;
    a.hq = hq;
    a.hkv = hkv;
    a.group = (int32_t)group;
    a.group_inv = 65536u / (uint32_t)group + 1;
    a.page_log2 = lp;
    a.num_pages = (int32_t)num_pages;
    a.prefix_len = prefix_len;
    a.slots = p.own_slots;
    a.max_tiles = p.max_tiles;
    a.o_f32 = o_dtype == TA_OUT_F32;
    const int score = (softcap > 0.f ? kScoreCap : 0) | (slopes ? kScoreSlope : 0);
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t err = hipSuccess;
    if (prefix) {
        PagedArgs b = a;
        b.slot_o = part(p.pre_slot_o);
        b.slot_lse = part(p.pre_slot_lse);
        b.row_o = part(p.pre_row_o);
        b.row_lse = part(p.pre_row_lse);
        b.slots = p.pre_slots;
        err = launch_pass<true>(head_dim, p.pre_rb, score, s, b);
    }
    if (err == hipSuccess)
        err = launch_pass<false>(head_dim, p.own_rb, score, s, a);
    if (err == hipSuccess) {
        JoinArgs j{};
        j.o = o;
        j.lse = lse;
        j.records = a.records;
        j.slot_o = a.slot_o;
        j.slot_lse = a.slot_lse;
        j.tile_rows = 32 * p.own_rb;
        j.chunk_rows = chunk_rows;
        j.chunks = chunks;
        j.row_o = a.row_o;
        j.row_lse = a.row_lse;
        j.pre_slot_o = part(p.pre_slot_o);
        j.pre_slot_lse = part(p.pre_slot_lse);
        j.pre_row_o = part(p.pre_row_o);
        j.pre_row_lse = part(p.pre_row_lse);
        j.prefix_len = prefix_len;
        j.pre_rows = 32 * p.pre_rb;
        const int step = p.pre_rb == 4 ? PagedShape<128, 4>::STEP : PagedShape<128, 1>::STEP;
        j.pre_steps = (prefix_len + step - 1) / step;
        j.pre_share =
            (int32_t)std::max<int64_t>(p.pre_rb == 4 ? PagedShape<128, 4>::LEAST
                                                     : PagedShape<128, 1>::LEAST,
                                       (pre_tiles * j.pre_steps + p.pre_slots - 1) / p.pre_slots);
        j.slopes = slopes;
        j.total_tokens = (int32_t)total_tokens;
        j.hq = hq;
        j.hkv = hkv;
        j.group = (int32_t)group;
        j.o_f32 = a.o_f32;
        const dim3 grid((uint32_t)(p.n_records * chunks * hkv));
        if (head_dim == 128)
            hipLaunchKernelGGL(paged_join_kernel<128>, grid, dim3(kJoinThreads), 0, s, j);
        else
            hipLaunchKernelGGL(paged_join_kernel<64>, grid, dim3(kJoinThreads), 0, s, j);
        err = hipGetLastError();
    }
    if (err != hipSuccess)
        return fail(TA_ERR_HIP, "%s: %s", fn, hipGetErrorString(err));
    return TA_OK;
}
