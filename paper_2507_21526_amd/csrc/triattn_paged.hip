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
//
// Both passes have a form for bf16 caches and forms for 8-bit ones (Q8): the latter
// convert K and V to bf16 where they are used, in registers for up to 32 rows, on
// their way into LDS for more, and multiply as the former do.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "triattn_device.h"
#include "triattn_internal.h"
#include "triattn_rows.h"
#include "triattn_rows8.h"
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
    const uint16_t *q;
    const unsigned char *kc, *vc;  // bf16, or 8-bit elements with
    const unsigned char *ks, *vs;  // a scale a row
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
    int32_t by_tile;  // whether a record belongs to each row tile, not to each share
    int32_t o_f32;
};

// Shapes of the two forms of the pass.
//   RB = 1: up to 32 rows, bound by the bytes of K and V.  Two waves take 32-key
//     tiles in turn, each into two stages of its own, and keep their own softmax:
//     nothing waits on the other wave until they are joined at the end of a
//     piece.  64 KB of stages at d = 128 (32 KB at d = 64) let two workgroups
//     (four) share a CU, so that one loads while the other finds its next request
//     or joins its waves.  The tables of lengths come on top, 16 to 20 bytes a
//     request with query offsets and 8 without: fewer bf16 workgroups share a CU from
//     some 700 requests with offsets on at d = 128, from 280 (700 without) at d = 64.
//   RB = 4: four waves of 32 rows each over the same 64-key tiles, in two stages.
//   RB = 0 (8-bit caches): as RB = 1, up to 16 rows.  The 8-bit forms of both take
//     64-key tiles (68 KB of stages, 34 KB at d = 64) and stream them through all row
//     tiles of a share.  With the query rows that leaves less for the tables: fewer
//     share a CU from some 310 requests of four tokens (group 4) on at d = 128, from 85
//     (single tokens without offsets: 443) at d = 64.
//   RB = 8 (8-bit caches): as RB = 4 with two groups of four waves, one wave of each on
//     a SIMD, in turns: the matrix products of one beside the softmax of the other.
template <int D, int RB, bool Q8>
struct PagedShape {
    static constexpr bool TILES8 = Q8 && RB <= 1;  // tiles in LDS hold 8 bits too
    static constexpr int NKB = RB >= 4 || TILES8 ? 2 : 1;
    static constexpr int TK = 32 * NKB;      // keys of a tile
    static constexpr int KS = RB >= 4 ? 1 : 2;  // key splits of a workgroup
    static constexpr int THREADS = 64 * (RB >= 4 ? RB : 1) * KS;
    static constexpr int STEP = TK * KS;     // keys of a step
    static constexpr int ROWS = RB == 0 ? 16 : 32 * RB;
    static constexpr int TILE_BYTES = TK * (TILES8 ? D : 2 * D);
    // K tile, V tile, and of 8-bit tiles the scales: the bytes as they come (K's,
    // V's), then V's as fp32
    static constexpr int STAGE_BYTES = 2 * TILE_BYTES + (TILES8 ? 512 : 0);
    static constexpr int STAGES = 2;
    static constexpr int BUFFER_BYTES = STAGES * STAGE_BYTES;  // of a wave (RB = 1)
    static constexpr int Q_BYTES = TILES8 ? ROWS * 2 * D : 0;  // the next piece's query rows
    static constexpr int LDS_BYTES = KS * BUFFER_BYTES + Q_BYTES;
    // What a row tile costs a share beside its steps, in steps (8-bit tiles): us of
    // 96 requests of 150 to 15000 keys (32 heads over 8, d = 128) with one 145, with
    // two 146, three 151; without, 179 where two took 156.
    static constexpr int CHARGE = TILES8 ? 1 : 0;
    // Least steps of a share: one of a 128-row tile leaves partials of twice
    // its K and V tiles' bytes.  us with 1, 4 and 8 steps (32 heads over 8, d =
    // 128): the last 64 tokens of 2000 27, 25, 29, of four times 1000 29, 25, 28,
    // 128 single tokens behind a prefix of 2048 47, 43, 44, the last 100 tokens of
    // 500 17, 24, 29; from 3000 keys on the same.
    // The 8-bit forms gain by any cut where there is little work: five requests of 4
    // to 14 tokens, 29 to 6462 keys behind a prefix of 76 (16 heads over 2, d = 128,
    // capped) with 4, 2 and 1 47, 37, 35, 100 tokens of 3000 (8 over 1) 37, 34, 31, the
    // 160 single tokens behind 10007 keys 88 with each.
    static constexpr int LEAST = RB >= 4 && !Q8 ? 4 : 1;
    static constexpr int WGS_PER_CU = RB == 8 ? 1 : RB <= 1 && D == 64 ? 4 : 2;
    static constexpr int WAVES_PER_SIMD = (WGS_PER_CU * THREADS / 64 + 3) / 4;
    // LDS of a workgroup beside the tables: stages and query rows, page ids, what the
    // waves of a piece and of the scan leave, the two flags
    static constexpr int FIXED_LDS = LDS_BYTES + 4 * (TILES8 ? 1 : kPageEntries) +
                                     KS * (12 + 256) + THREADS / 16 + 8;
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

template <int D, int RB, int SCORE, bool PREFIX, bool Q8>
__global__ __launch_bounds__((PagedShape<D, RB, Q8>::THREADS),
                             (PagedShape<D, RB, Q8>::WAVES_PER_SIMD)) void paged_attn_kernel(PagedArgs a)
{
    using S = PagedShape<D, RB, Q8>;
    constexpr int kThreads = S::THREADS;
    constexpr int ROW_BYTES = Q8 ? D : 2 * D;            // of a cached row
    constexpr int CHUNKS = ROW_BYTES / 16;
    constexpr int COPY_ROWS = 1024 / ROW_BYTES;          // keys of a 1 KB copy
    constexpr int GROUP = 16;  // keys that surely share a page
    constexpr int COPIES = GROUP / COPY_ROWS;              // 1 KB copies of a group
    constexpr int GROUPS = S::TK / GROUP / (RB >= 4 ? 4 : 1);  // of a wave and tile
    constexpr int D_BLOCKS = D / 32;

    __shared__ __attribute__((aligned(1024))) unsigned char smem[S::LDS_BYTES];
    // tables of the own-keys pass, as long as the call needs (table_bytes)
    extern __shared__ int32_t tables[];
    int32_t *const s_step = tables;                   // first step of a row tile, and the total
    int32_t *const s_kv = s_step + a.max_tiles + 1;   // own keys of a request
    int32_t *const s_req = s_kv + a.batch;            // first row tile of a request, and all
    int32_t *const s_cu = s_req + a.batch + 1;        // query offsets
    __shared__ int32_t s_page[S::TILES8 ? 1 : kPageEntries];
    __shared__ int32_t s_end[S::KS][3];  // of a wave's piece: bad key, odd values, free stage
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
            const int steps = (tile_of(t).limit + S::STEP - 1) / S::STEP;
            return steps > 0 ? steps + S::CHARGE : 0;
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
            // one share's row tile needs no join, unless a prefix's rows do
            const bool cut =
                (s_step[t] + S::CHARGE) / share != (s_step[t + 1] - 1) / share;
            m[RF_Q0] = r.q0;
            m[RF_RHO0] = r.rho0;
            m[RF_ROWS] = cut || a.row_o ? r.rows : 0;
            m[RF_POS0] = r.pos0;
            m[RF_BEGIN] = s_step[t];
            m[RF_END] = s_step[t + 1];
            m[RF_SHARE] = share;
        };
        if (g == 0 && a.by_tile) {
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
    const int wave_lds = RB <= 1 ? wave * S::BUFFER_BYTES : 0;
    const int first_group = RB <= 1 ? 0 : (wave & 3) * GROUPS;
    const int dma_row = lane / CHUNKS;
    // a copying lane's place in a group's first block; block m flips the K
    // swizzle's bits of m COPY_ROWS
    const uint32_t dma_k = (uint32_t)(
        dma_row * ROW_BYTES +
        (((lane % CHUNKS) ^ (Q8 ? rows8_swz<D>(dma_row) : rows_kswz<D>(dma_row))) << 4));
    const uint32_t dma_v =
        Q8 ? dma_k
           : (uint32_t)(dma_row * ROW_BYTES + (((lane % CHUNKS) ^ rows_vswz<D>(dma_row)) << 4));
    const int64_t page_stride = ((int64_t)a.hkv << a.page_log2) * ROW_BYTES;
    const int64_t head_off = ((int64_t)g << a.page_log2) * ROW_BYTES;
    const unsigned char *kc = a.kc + head_off;
    const unsigned char *vc = a.vc + head_off;
    const int page_mask = (1 << a.page_log2) - 1;
    // the scale of a key of this head in a page
    auto scale_at = [&](const unsigned char *base, int id, int place) TA_INLINE {
        return base + ((((int64_t)id * a.hkv + g) << a.page_log2) + place);
    };

    std::conditional_t<S::TILES8,
                       std::conditional_t<RB == 0, RowBlock8x16<D, S::NKB, SCORE>,
                                          RowBlock8<D, S::NKB, SCORE>>,
                       RowBlock<D, S::NKB, SCORE>>
        rb;
    rb.init(lane);

    if constexpr (S::TILES8) {
        // One stream of tiles through all pieces of the share: a wave's copies run
        // STAGES tiles ahead of its products, into the next piece too, so that the
        // latencies of page ids (which scalar loads bring a tile ahead of the
        // copies), query rows and first tiles are not paid anew at every request.
        constexpr bool BACK = (SCORE & kScoreSlope) != 0;  // last keys first, see below
        constexpr int V_COPIES = GROUPS * COPIES, K_COPIES = V_COPIES + 1;  // K's: scales too
        constexpr int Q_COPIES = S::Q_BYTES / 1024 / S::KS;  // of a wave
        constexpr int HALF = decltype(rb)::CHUNKS / 2;
        const uint32_t q_lds = smem_addr + S::KS * S::BUFFER_BYTES;
        typedef const __attribute__((address_space(4))) int32_t *ids_ptr;

        struct Piece {
            RowTile rt;
            int tile;          // which row tile
            int begin, cost;   // of it, in the shares' units
            int step0, step1;  // of the row tile
            int base, n;       // this wave's tiles: first key of the first one, how many
            int slot;          // of the partials; -1: the whole row tile
        };
        // the first piece from `at` on; n_tiles' end: none
        auto open = [&](int at, int t, Piece &p) TA_INLINE -> bool {
            for (;;) {
                if (at >= share1)
                    return false;
                if constexpr (PREFIX) {
                    t = at / prefix_steps;
                    p.begin = t * prefix_steps;
                    p.cost = prefix_steps;
                } else {
                    if (t < 0)
                        t = find_start(s_step, n_tiles, at);
                    else
                        do
                            ++t;
                        while (s_step[t + 1] <= at);
                    t = uni(t);
                    p.begin = uni(s_step[t]);
                    p.cost = uni(s_step[t + 1]) - p.begin;
                }
                constexpr int C = PREFIX ? 0 : S::CHARGE;
                p.step0 = max(0, at - p.begin - C);
                p.step1 = min(share1, p.begin + p.cost) - p.begin - C;
                if (p.step1 > p.step0)
                    break;
                at = p.begin + p.cost;  // the share ends within the row tile's charge
                if (at < share1)
                    continue;
                return false;
            }
            p.rt = tile_of(t);
            p.rt.q0 = uni(p.rt.q0);
            p.rt.rho0 = uni(p.rt.rho0);
            p.rt.rows = uni(p.rt.rows);
            p.rt.pos0 = uni(p.rt.pos0);
            p.rt.limit = uni(p.rt.limit);
            p.rt.req = uni(p.rt.req);
            p.tile = t;
            p.base = p.step0 * S::STEP + wave * S::TK;
            const int end = min(p.step1 * S::STEP, p.rt.limit);
            p.n = p.base < end ? (end - p.base + S::STEP - 1) / S::STEP : 0;
            p.slot = p.step0 == 0 && p.step1 == p.cost - (PREFIX ? 0 : S::CHARGE)
                         ? -1
                         : 2 * slot + (p.begin > share0 ? 1 : 0);
            return true;
        };
        auto after = [&](const Piece &p, Piece &q) TA_INLINE -> bool {
            return open(p.begin + p.cost, p.tile, q);
        };
        auto key_of = [&](int base, int n, int i) TA_INLINE -> int {
            return base + (BACK ? n - 1 - i : i) * S::STEP;
        };
        auto pages_of = [&](const Piece &p) TA_INLINE -> ids_ptr {
            return (ids_ptr)(uintptr_t)(PREFIX ? a.prefix_pages
                                               : a.table + (int64_t)p.rt.req * a.width);
        };

        // The pages of a tile's groups of keys.
        using Ids = int[GROUPS];
        auto find_ids = [&](ids_ptr ids, int limit, int key0, Ids &id) TA_INLINE {
#pragma unroll
            for (int i = 0; i < GROUPS; ++i)
                id[i] = ids[min(key0 + i * GROUP, limit - 1) >> a.page_log2];
        };
        // Page ids that are none become 0; returns the first key of such a page.
        auto check_ids = [&](int limit, int key0, Ids &id) TA_INLINE -> int {
            int bad = INT32_MAX;
#pragma unroll
            for (int i = 0; i < GROUPS; ++i) {
                id[i] = uni(id[i]);
                if ((uint32_t)id[i] >= (uint32_t)a.num_pages) {
                    id[i] = 0;
                    bad = min(bad, min(key0 + i * GROUP, limit - 1) & ~page_mask);
                }
            }
            return bad;
        };
        // Copies a tile's K rows and scales, or its V rows, into a stage.  Keys from
        // rt.limit on repeat the last one before it; they lie past every row's last
        // key.
        auto copy_part = [&](int limit, int key0, const Ids &id, int stage, auto is_v) TA_INLINE {
            constexpr bool V = decltype(is_v)::value;
            const uint32_t lds = smem_addr + wave_lds + stage * S::STAGE_BYTES;
            const bool inside = key0 + S::TK <= limit;
            asm volatile("" ::: "memory");
#pragma unroll
            for (int i = 0; i < GROUPS; ++i) {
                const int key = key0 + i * GROUP;
                const unsigned char *page = (V ? vc : kc) + (int64_t)uni(id[i]) * page_stride;
                const uint32_t to = lds + (V ? S::TILE_BYTES : 0) + i * GROUP * D;
                if (inside) {
                    const unsigned char *from = page + (key & page_mask) * D;
                    if constexpr (COPIES == 1) {
                        copy_to_lds16(from, dma_k, to);
                    } else {
                        const uint32_t off[2] = {dma_k, dma_k};
                        copy_burst_to_lds16<2>(from, off, to);
                    }
                } else {
#pragma unroll
                    for (int m = 0; m < COPIES; ++m) {
                        const int first = min(key + m * COPY_ROWS, limit - 1);
                        const int lim = limit - 1 - first;  // rows after the first
                        copy_to_lds16(page + (first & page_mask) * D,
                                      dma_k - (uint32_t)(max(dma_row - lim, 0) * D),
                                      to + m * 1024);
                    }
                }
            }
            // The scales: lane i copies four bytes, of K's keys or of V's (lanes
            // past them repeat the same).
            if constexpr (!V) {
                constexpr int PER = S::TK / 4;  // lanes of K's keys
                // (keys from the limit on: bytes of the last ones, not used)
                const int key = min(key0 + 4 * (lane & (PER - 1)), (limit - 1) & ~3);
                int mine = id[0];
#pragma unroll
                for (int i = 1; i < GROUPS; ++i)
                    mine = key >= key0 + i * GROUP ? id[i] : mine;
                copy_to_lds4(scale_at(lane & PER ? a.vs : a.ks, mine, key & page_mask),
                             lds + 2 * S::TILE_BYTES);
            }
            asm volatile("" ::: "memory");
        };
        using K = std::false_type;
        using V = std::true_type;
        // This wave's half of the copies of a piece's query rows (rows past the
        // tile repeat its last one), 16-byte chunks permuted by the row.
        constexpr int Q_CHUNKS = D / 8, Q_ROWS = 64 / Q_CHUNKS;  // of a 1 KB copy
        auto copy_q = [&](const Piece &p) TA_INLINE {
            asm volatile("" ::: "memory");
#pragma unroll
            for (int m = 0; m < Q_COPIES; ++m) {
                const int r = (wave * Q_COPIES + m) * Q_ROWS + lane / Q_CHUNKS;
                const int rho = p.rt.rho0 + min(r, p.rt.rows - 1), tq = div_group(rho);
                const int head = g * a.group + rho - tq * a.group;
                copy_to_lds16_at(a.q + ((int64_t)(p.rt.q0 + tq) * a.hq + head) * D +
                                     8 * ((lane % Q_CHUNKS) ^ (r & (Q_CHUNKS - 1))),
                                 q_lds + (wave * Q_COPIES + m) * 1024);
            }
            asm volatile("" ::: "memory");
        };
        auto read_q = [&]() TA_INLINE {
            const unsigned char *row = smem + S::KS * S::BUFFER_BYTES + rb.col * 2 * D;
#pragma unroll
            for (int i = 0; i < decltype(rb)::Q_FRAGMENTS; ++i)
                rb.qf[i] = *reinterpret_cast<const bf16x8 *>(
                    row + ((rb.q_chunk(i) ^ (rb.col & (Q_CHUNKS - 1))) << 4));
        };

        Piece cur, nxt;
        if (!open(share0, -1, cur))
            return;
        bool ahead = false;  // the copies are in nxt, not in cur
        bool q_due = false;  // nxt's query rows are not on their way yet
        bool has = false;    // there is a next tile, from key nt_key on
        int made = 0;        // tiles of the piece being copied, the next one among them
        int flying = 0;      // tiles whose copies have begun, not yet multiplied
        int in_stage = 0, out_stage = 0;
        int bad_cur = INT32_MAX, bad_nxt = INT32_MAX;
        int nt_key = 0;
        Ids nt;  // their pages (on their way)
        // of the piece being copied
        int src_base = cur.base, src_n = cur.n, src_limit = cur.rt.limit;
        ids_ptr src_pages = pages_of(cur);
        auto advance = [&]() TA_INLINE {
            has = false;
            if (made == src_n) {
                // at most one piece ahead: there is room for the rows of one
                if (ahead || !after(cur, nxt))
                    return;
                ahead = q_due = true;
                made = 0;
                src_base = nxt.base;
                src_n = nxt.n;
                src_limit = nxt.rt.limit;
                src_pages = pages_of(nxt);
                if (src_n == 0)
                    return;
            }
            nt_key = key_of(src_base, src_n, made);
            find_ids(src_pages, src_limit, nt_key, nt);
            ++made;
            has = true;
        };
        auto send_q = [&]() TA_INLINE {
            if (q_due)
                copy_q(nxt);
            q_due = false;
        };
        // The copies of the next tile: K's where the stage's K has been multiplied,
        // V's where its V has.
        auto produce_k = [&]() TA_INLINE {
            send_q();
            if (!has)
                return;
            const int bad = check_ids(src_limit, nt_key, nt);
            bad_nxt = ahead ? min(bad_nxt, bad) : bad_nxt;
            bad_cur = ahead ? bad_cur : min(bad_cur, bad);
            copy_part(src_limit, nt_key, nt, in_stage, K{});
        };
        auto produce_v = [&]() TA_INLINE {
            if (!has)
                return;
            copy_part(src_limit, nt_key, nt, in_stage, V{});
            in_stage = in_stage + 1 == S::STAGES ? 0 : in_stage + 1;
            ++flying;
            advance();
        };
        // until the K, and what was sent before it, of the oldest tile has come; its
        // V (behind it the next tile, and K of the one after where `more`)
        static_assert(S::STAGES == 2, "what may be behind a tile");
        auto wait_k = [&]() TA_INLINE {
            if (flying >= 2)
                rows_wait_copies<2 * V_COPIES + K_COPIES>();
            else if (flying == 1)
                rows_wait_copies<V_COPIES>();
            else
                rows_wait_copies<0>();
        };
        auto wait_v = [&](bool more) TA_INLINE {
            if (flying >= 2 && more)
                rows_wait_copies<V_COPIES + 2 * K_COPIES>();
            else if (flying >= 2)
                rows_wait_copies<V_COPIES + K_COPIES>();
            else
                rows_wait_copies<0>();
        };
        copy_q(cur);
        advance();
        while (has && !ahead && flying < S::STAGES) {
            produce_k();
            produce_v();
        }
        wait_k();
        barrier_no_fence();
        read_q();
        barrier_no_fence();  // its place is free

        for (;;) {
            while (has && flying < S::STAGES) {
                produce_k();
                produce_v();
            }
            // this lane's query row (rows past the tile repeat its last one)
            const RowTile rt = cur.rt;
            const int rho = rt.rho0 + min(rb.col, rt.rows - 1);
            const int tq = div_group(rho);
            const int head = g * a.group + rho - tq * a.group;
            float slope = 0.f;
            if constexpr ((SCORE & kScoreSlope) != 0)
                slope = a.score.slopes[head] * kRowsLog2e;
            // as in the other forms: the last key that this row keeps, and the
            // first row's; and where distances are taken from
            const int last = PREFIX ? a.prefix_len - 1 : rt.pos0 + tq;
            const int first_last = PREFIX ? a.prefix_len - 1 : rt.pos0 + div_group(rt.rho0);
            int dist_row = PREFIX ? a.prefix_len : last;
            if constexpr ((SCORE & kScoreSlope) != 0)
                if (slope < 0.f)
                    dist_row = PREFIX ? 0 : -a.prefix_len;
            bool fresh = true, odd = false;
            bool refilled = false;  // K of the tile after the next is on its way
            rb.reset();
            // between(): after the products with K
            auto tile = [&](int key0, unsigned char *kt, auto careful, auto &&between)
                            TA_INLINE {
                constexpr bool CAREFUL = decltype(careful)::value;
                // V's scales as fp32 in kWeightUnit, 0 for a key that no row keeps
                static_assert(S::TK == 64, "a key a lane");
                unsigned char *raw = kt + 2 * S::TILE_BYTES;
                const uint32_t byte = raw[S::TK + lane];
                const bool on = key0 + lane < rt.limit;
                float *vscale = reinterpret_cast<float *>(raw + 256);
                vscale[lane] = on ? kWeightUnit * q8_scale(byte) : 0.f;
                typename decltype(rb)::Scores s;
                typename decltype(rb)::Probs p;
                rb.products8(kt, raw, s);
                between();
                rb.modify(s, a.score);
                const bool masked = key0 + S::TK - 1 > first_last;
                if (__builtin_expect(masked, 0)) {
                    asm volatile("");  // a branch: most tiles have no mask
                    rb.mask_above(s, last - key0);
                }
                rb.softmax8(s, a.score, slope, key0 - dist_row, p, fresh, vscale);
                fresh = false;
                if constexpr (CAREFUL) {
                    rb.accumulate8_by_key(kt + S::TILE_BYTES, s, p);
                } else {
                    wait_v(refilled);
                    if (__builtin_expect(masked, 0)) {
                        asm volatile("");
                        odd |= __builtin_amdgcn_ballot_w64(on && byte == 255) != 0 ||
                               rows8_odd_elements<S::TILE_BYTES>(kt + S::TILE_BYTES, lane);
                    }
                    rb.accumulate8(kt + S::TILE_BYTES, p);
                }
            };
            for (int i = 0; i < cur.n; ++i) {
                wait_k();
                // every read of a stage has returned before it is written again;
                // the last tile's stage joins the waves first
                refilled = i + 1 < cur.n && has;
                tile(key_of(cur.base, cur.n, i), smem + wave_lds + out_stage * S::STAGE_BYTES,
                     std::false_type{}, [&]() TA_INLINE {
                         if (i + 1 < cur.n) {
                             __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
                             produce_k();
                         }
                     });
                out_stage = out_stage + 1 == S::STAGES ? 0 : out_stage + 1;
                --flying;
                if (i + 1 < cur.n) {
                    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
                    produce_v();
                }
            }
            const int free_stage = (out_stage + S::STAGES - 1) % S::STAGES;
            unsigned char *const scratch = smem + wave_lds + free_stage * S::STAGE_BYTES;

            // The waves join, each finishing half of the d blocks: it leaves the
            // other half of its sums in its free stage.
            static_assert(HALF * 1024 <= S::STAGE_BYTES, "half of the sums fit a stage");
            auto leave = [&](int odd_values) TA_INLINE {
                const float l = rb.row_sum(rb.l_run);
                if (rb.first()) {
                    s_ml[wave][rb.col][0] = rb.m_ref;
                    s_ml[wave][rb.col][1] = l;
                }
                if (lane == 0) {
                    s_end[wave][0] = bad_cur;
                    s_end[wave][1] = odd_values;
                    s_end[wave][2] = free_stage;
                }
                if (cur.n == 0)
                    return;
#pragma unroll
                for (int c = 0; c < HALF; ++c)
                    *reinterpret_cast<f32x4r *>(scratch + (c * 64 + lane) * 16) =
                        wave ? rb.chunk(c) : rb.chunk(HALF + c);
            };
            leave(odd);
            if (!ahead && !has)
                advance();
            send_q();
            wait_k();  // nxt's first keys, and its query rows before them
            barrier_no_fence();
            if (__builtin_expect(s_end[0][1] | s_end[1][1], 0)) {
                // a masked tile holds NaN values: the piece again, tile by tile in
                // the free stage, each key only to the rows that keep it
                barrier_no_fence();
                fresh = true;
                rb.reset();
                for (int i = 0; i < cur.n; ++i) {
                    const int key0 = key_of(cur.base, cur.n, i);
                    Ids id;
                    find_ids(pages_of(cur), rt.limit, key0, id);
                    check_ids(rt.limit, key0, id);
                    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
                    copy_part(rt.limit, key0, id, free_stage, K{});
                    copy_part(rt.limit, key0, id, free_stage, V{});
                    rows_wait_copies<0>();
                    tile(key0, scratch, std::true_type{}, []() {});
                }
                leave(0);
                barrier_no_fence();
            }
            const int bad_key = min(s_end[0][0], s_end[1][0]);
            const float m0 = s_ml[0][rb.col][0], m1 = s_ml[1][rb.col][0];
            const float m = fmaxf(m0, m1), m_use = m == -INFINITY ? 0.f : m;
            const float f0 = __builtin_amdgcn_exp2f(m0 - m_use);
            const float f1 = __builtin_amdgcn_exp2f(m1 - m_use);
            const float den = f0 * s_ml[0][rb.col][1] + f1 * s_ml[1][rb.col][1];
            // NaN from the first page that is none on (earlier rows of the tile do
            // not keep its keys)
            const float nan = last >= bad_key ? __builtin_nanf("") : 0.f;
            const float inv = (den == 0.f ? 0.f : (1.f / kWeightUnit) / den) + nan;
            const bool to_o = cur.slot < 0 && !a.row_o;
            const int64_t orow = (int64_t)(rt.q0 + tq) * a.hq + head;
            const int64_t srow = ((int64_t)cur.slot * a.hkv + g) * S::ROWS + rb.col;
            const unsigned char *theirs = smem + (1 - wave) * S::BUFFER_BYTES +
                                          s_end[1 - wave][2] * S::STAGE_BYTES;
            // (sums that the other wave left nowhere, having no tile, are zero)
            const bool other = (wave ? m0 : m1) != -INFINITY;
            if (rb.col < rt.rows) {
#pragma unroll
                for (int c = 0; c < HALF; ++c) {
                    f32x4r x{};
                    if (other)
                        x = *reinterpret_cast<const f32x4r *>(theirs + (c * 64 + lane) * 16);
                    const f32x4r mine = wave ? rb.chunk(HALF + c) : rb.chunk(c);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        x[e] = (f0 * (wave ? x[e] : mine[e]) + f1 * (wave ? mine[e] : x[e])) * inv;
                    const int d0 = rb.chunk_d(wave * HALF + c);
                    if (to_o && !a.o_f32)
                        *reinterpret_cast<bf16x4r *>(static_cast<__bf16 *>(a.o) + orow * D + d0) =
                            __builtin_convertvector(x, bf16x4r);
                    else if (to_o)
                        *reinterpret_cast<f32x4r *>(static_cast<float *>(a.o) + orow * D + d0) = x;
                    else
                        *reinterpret_cast<f32x4r *>(cur.slot < 0 ? a.row_o + orow * D + d0
                                                                 : a.slot_o + srow * D + d0) = x;
                }
                if (wave == 0 && rb.first()) {
                    float lse = (den == 0.f ? -INFINITY : (m + __log2f(den)) * kRowsLn2) + nan;
                    if (to_o) {
                        if constexpr ((SCORE & kScoreSlope) != 0)
                            lse += rows_lse_shift(a.score.slopes[head], rt.pos0 + tq);
                        if (a.lse)
                            a.lse[(int64_t)head * a.total_tokens + rt.q0 + tq] = lse;
                    } else if (cur.slot < 0) {
                        a.row_lse[orow] = lse;
                    } else {
                        a.slot_lse[srow] = lse;
                    }
                }
            }
            if (!ahead)
                return;
            cur = nxt;
            ahead = false;
            bad_cur = bad_nxt;
            bad_nxt = INT32_MAX;
            read_q();
            barrier_no_fence();  // the free stages and the rows' place are read
            if (!has)
                advance();
        }
    } else {
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
                if constexpr (Q8) {
                    __builtin_amdgcn_s_setprio(1);
                    rb.template in_order<false, true>(vt, vt, s, p);
                    __builtin_amdgcn_s_setprio(0);
                } else {
                    __builtin_amdgcn_sched_barrier(0);
                    rb.accumulate(vt, p);
                    rb.template schedule<false, true>();
                    __builtin_amdgcn_sched_barrier(0);
                }
            };
            auto products = [&](const unsigned char *kt) TA_INLINE {
                if constexpr (Q8) {
                    rb.template in_order<true, false>(kt, kt, s, p);
                } else {
                    __builtin_amdgcn_sched_barrier(0);
                    rb.products(kt, s);
                    rb.template schedule<true, false>();
                    __builtin_amdgcn_sched_barrier(0);
                }
            };
            // An 8-bit cache's rows as bf16 tiles: a wave loads a group's rows and
            // scales into registers, and later leaves them in LDS, each element times
            // its scale.  With eight waves the first four take K, the others V.
            constexpr int LOADS = Q8 ? GROUP * D / 1024 : 1;  // 16-byte loads of a lane, K or V
            constexpr int LOAD_ROWS = GROUP / LOADS;
            constexpr int TENSORS = RB == 8 ? 1 : 2;
            const int group = wave & 3, tensor0 = RB == 8 ? wave >> 2 : 0;
            u32x4 held[TENSORS][LOADS];
            uint32_t held_scale[TENSORS][LOADS];
            const int load_row = lane / (D / 16), load_chunk = lane % (D / 16);
            auto load_rows = [&](int key0) TA_INLINE {
                const int first = min(key0 + group * GROUP, rt.limit - 1);
                const int lim = min(rt.limit - 1 - first, GROUP - 1);  // the group's last row
                const int id = uni(s_page[(first >> a.page_log2) - page0]);
                const int place = first & page_mask;
                const int64_t off = (int64_t)id * page_stride + place * ROW_BYTES;
#pragma unroll
                for (int v = 0; v < TENSORS; ++v) {
                    const unsigned char *rows = (tensor0 + v ? vc : kc) + off;
                    const unsigned char *scale = scale_at(tensor0 + v ? a.vs : a.ks, id, place);
#pragma unroll
                    for (int m = 0; m < LOADS; ++m) {
                        const uint32_t row = min(m * LOAD_ROWS + load_row, lim);
                        held[v][m] = *reinterpret_cast<const u32x4 *>(
                            rows + (row * D + load_chunk * 16));
                        held_scale[v][m] = scale[row];
                    }
                }
            };
            auto leave_rows = [&](int c, int stage) TA_INLINE {
                const int v = c / LOADS, m = c % LOADS;
                const int row = m * LOAD_ROWS + load_row;  // in the group
                const int swz = tensor0 + v ? rows_vswz<D>(row) : rows_kswz<D>(row);
                const uint32_t to = smem_addr + stage * S::STAGE_BYTES +
                                    (tensor0 + v) * S::TILE_BYTES + (group * GROUP + row) * 2 * D;
                const float f = q8_scale_bits(held_scale[v][m]);
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    write_lds16(to + (((2 * load_chunk + i) ^ swz) << 4),
                                q8_fragment(held[v][m][2 * i], held[v][m][2 * i + 1], f));
            };
            auto leave_all = [&](int stage) TA_INLINE {
                asm volatile("" ::: "memory");
#pragma unroll
                for (int c = 0; c < TENSORS * LOADS; ++c)
                    leave_rows(c, stage);
                asm volatile("" ::: "memory");
            };
            if constexpr (CAREFUL) {
                // tile by tile, in this wave's first stage (RB = 1) or the
                // workgroup's
                const int n = (key_end - seg0 * S::STEP + S::STEP - 1) / S::STEP;
                for (int i = 0; i < n; ++i) {
                    const int key0 = (seg0 + (BACK ? n - 1 - i : i)) * S::STEP +
                                     (RB == 1 ? wave * S::TK : 0);
                    const bool on = key0 < key_end;
                    if constexpr (Q8) {
                        load_rows(key0);
                        leave_all(0);
                    } else if (on) {
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
            } else if constexpr (RB == 8) {
                // M(j) = {S(j) = K(j) Q^T, O += V(j - 1) P(j - 1)} on the matrix cores
                // beside the other group's X(j), scores to probabilities, on the vector
                // units.  Both groups run the same program, group 1 a phase later:
                // group 0 has M(j) in phase 2 j and X(j) in phase 2 j + 1.  Stage j & 1
                // holds K(j) and V(j - 1) in the two phases of M(j).  In X(j), after the
                // softmax, group 0 leaves K(j + 1) in stage (j + 1) & 1 and group 1
                // V(j + 1) in stage j & 1, which no wave reads any more by then, and loads
                // the rows of step j + 2; nothing but LDS reads stands between the matrix
                // instructions of M(j).
                const int n = (key_end - seg0 * S::STEP + S::STEP - 1) / S::STEP;
                auto key_of = [&](int i) TA_INLINE -> int {
                    i = min(i, n - 1);
                    return (seg0 + (BACK ? n - 1 - i : i)) * S::STEP;
                };
                auto end_phase = [&]() TA_INLINE {
                    __builtin_amdgcn_sched_barrier(0);
                    barrier_no_fence();
                    __builtin_amdgcn_sched_barrier(0);
                };
                auto matrix = [&](int j, auto stage) TA_INLINE {
                    const unsigned char *kt = smem + decltype(stage)::value * S::STAGE_BYTES;
                    if (__builtin_expect(key_of(j - 1) + S::TK - 1 > tile_first_last, 0)) {
                        asm volatile("");
                        odd |= rb.odd_values(kt + S::TILE_BYTES, lane, wave, RB);
                    }
                    __builtin_amdgcn_s_setprio(1);
                    rb.template in_order<true, true>(kt, kt + S::TILE_BYTES, s, p);
                    __builtin_amdgcn_s_setprio(0);
                };
                // (past the last step its rows once more, where nothing reads them)
                auto vector = [&](int j) TA_INLINE {
                    softmax(key_of(j));
                    __builtin_amdgcn_sched_barrier(0);
                    leave_all(tensor0 ? j & 1 : (j + 1) & 1);
                    load_rows(key_of(j + 2));
                };
                load_rows(key_of(0));
                leave_all(tensor0);
                load_rows(key_of(1));
                end_phase();
                if (tensor0)
                    end_phase();
                products(smem);
                end_phase();
                vector(0);
                end_phase();
                auto step = [&](int j, auto stage) TA_INLINE {
                    matrix(j, stage);
                    end_phase();
                    vector(j);
                    end_phase();
                };
                int j = 1;
                for (; j + 1 < n; j += 2) {
                    step(j, std::integral_constant<int, 1>{});
                    step(j + 1, std::integral_constant<int, 0>{});
                }
                if (j < n)
                    step(j, std::integral_constant<int, 1>{});
                values(key_of(n - 1), smem + (n & 1) * S::STAGE_BYTES + S::TILE_BYTES);
                end_phase();
                if (!tensor0)
                    end_phase();
            } else if constexpr (Q8) {
                // As below, but through registers: step i leaves the rows of step
                // i + 1 in LDS after its products, and then loads those of i + 2.
                const int n = (key_end - seg0 * S::STEP + S::STEP - 1) / S::STEP;
                auto key_of = [&](int i) TA_INLINE -> int {
                    return (seg0 + (BACK ? n - 1 - i : i)) * S::STEP;
                };
                load_rows(key_of(0));
                leave_all(0);
                load_rows(key_of(min(1, n - 1)));
                auto step = [&](int i, auto stage) TA_INLINE {
                    constexpr int ST = decltype(stage)::value;
                    // this step's tile is there for every wave, and every wave is
                    // done with the other stage
                    __builtin_amdgcn_sched_barrier(0);
                    barrier_no_fence();
                    const unsigned char *kt = smem + ST * S::STAGE_BYTES;
                    __builtin_amdgcn_s_setprio(1);
                    products(kt);
                    __builtin_amdgcn_s_setprio(0);
                    // (after the last step its tile is left once more, in the stage
                    // that nothing reads any more)
                    leave_all(1 - ST);
                    load_rows(key_of(min(i + 2, n - 1)));
                    __builtin_amdgcn_sched_barrier(0);
                    softmax(key_of(i));
                    values(key_of(i), kt + S::TILE_BYTES);
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
            static_assert(32 * PITCH <= S::BUFFER_BYTES, "accumulators fit the wave's stages");
            auto place = [&](int r, int chunk) TA_INLINE -> int {
                return r * PITCH + ((chunk ^ (r & (D / 4 - 1))) << 4);
            };
            unsigned char *mine = smem + wave * S::BUFFER_BYTES;
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
                        smem + w * S::BUFFER_BYTES + place(r, d0 / 4));
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
}

struct JoinArgs {
    void *o;
    float *lse;
    const int32_t *records;
    const float *slot_o, *slot_lse;
    int32_t tile_rows;
    int32_t chunks, chunk_rows;  // workgroups of a row tile, rows of each
    int32_t ways;                // groups of lanes of a row
    int32_t charge;              // of a row tile beside its steps
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
// to a row 50).  Where few requests share the chip a row has many partials: WIDE
// then gives it `ways` groups of sixteen lanes, which take every ways-th partial each
// and join in LDS (three requests of 128K keys, 43 partials a row: 6.4 us, one way 22).
template <int D, bool WIDE>
__global__ __launch_bounds__(kJoinThreads) void paged_join_kernel(JoinArgs a)
{
    constexpr int LANES = 16;        // of a row
    constexpr int PER = D / LANES;   // values of a lane, in runs of four
    constexpr int RUNS = PER / 4;
    constexpr int GROUPS = kJoinThreads / LANES;
    __shared__ __attribute__((aligned(16))) float s_part[WIDE ? GROUPS : 1][WIDE ? D + 4 : 4];
    const int ways = WIDE ? a.ways : 1;
    const int g = blockIdx.x % a.hkv, at = blockIdx.x / a.hkv;
    const int chunk = at % a.chunks;
    const int32_t *m = a.records + kRecordWords * (at / a.chunks);
    const int32_t q0 = m[RF_Q0], rho0 = m[RF_RHO0], rows = m[RF_ROWS], pos0 = m[RF_POS0];
    const int32_t begin = m[RF_BEGIN], end = m[RF_END], share = m[RF_SHARE];
    if (rows == 0)
        return;
    const int w0 = (begin + a.charge) / share;
    const int n_own = (end - 1) / share - w0 + 1;
    const int lane = threadIdx.x % LANES;
    {
        const int way = threadIdx.x / LANES % ways;
        int r = chunk * a.chunk_rows + threadIdx.x / LANES / ways;
        const bool mine = (int)(threadIdx.x / LANES) < a.chunk_rows * ways && r < rows;
        if constexpr (!WIDE) {
            if (!mine)
                return;
        } else {
            r = min(r, rows - 1);  // (lanes past the rows wait for the others)
        }
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
        // this way's partials: way, way + ways, ..
        const int all = n_pre + n_own;
        const int n = WIDE ? max(0, all - way + ways - 1) / ways : all;
        // row of partial c: in the whole rows or the pieces of its pass
        auto index = [&](int i) TA_INLINE -> int64_t {
            const int c = WIDE ? way + ways * i : i;
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
        auto lse_of = [&](int i) TA_INLINE -> float {
            const int c = WIDE ? way + ways * i : i;
            const float *from = c < n_pre ? (n_pre == 1 ? a.pre_row_lse : a.pre_slot_lse)
                                          : (n_own == 1 ? a.row_lse : a.slot_lse);
            return from[index(i)] + (c < n_pre ? shift : 0.f);
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
                    const int i = c0 + min(c + u, top - 1), cc = WIDE ? way + ways * i : i;
                    const float *from = cc < n_pre ? (n_pre == 1 ? a.pre_row_o : a.pre_slot_o)
                                                   : (n_own == 1 ? a.row_o : a.slot_o);
                    from += index(i) * D + 4 * lane;
#pragma unroll
                    for (int k = 0; k < RUNS; ++k)
                        x[u][k] = *reinterpret_cast<const f32x4r *>(from + 4 * LANES * k);
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
        float m_all = m_use;
        if constexpr (WIDE) {
            // the ways of a row, in order
            float *const to = s_part[threadIdx.x / LANES];
#pragma unroll
            for (int i = 0; i < RUNS; ++i)
                *reinterpret_cast<f32x4r *>(to + 4 * LANES * i + 4 * lane) = acc[i];
            if (lane == 0) {
                to[D] = n > 0 ? mx : -INFINITY;
                to[D + 1] = den;
            }
            __syncthreads();
            if (!mine || way != 0)
                return;
            const float(*part)[D + 4] = &s_part[threadIdx.x / LANES];
            float top = -INFINITY;
            for (int w = 0; w < ways; ++w)
                top = fmaxf(top, part[w][D]);
            m_all = top == -INFINITY ? 0.f : top;
            den = 0.f;
#pragma unroll
            for (int i = 0; i < RUNS; ++i)
                acc[i] = f32x4r{};
            for (int w = 0; w < ways; ++w) {
                const float f = __expf(part[w][D] - m_all);
                den += f * part[w][D + 1];
#pragma unroll
                for (int i = 0; i < RUNS; ++i) {
                    const f32x4r y =
                        *reinterpret_cast<const f32x4r *>(part[w] + 4 * LANES * i + 4 * lane);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        acc[i][e] += f * y[e];
                }
            }
        }
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
                           : m_all + __logf(den) +
                                 (a.slopes ? rows_lse_shift(a.slopes[h], a.prefix_len + pos0 + qt)
                                           : 0.f);
    }
}

// How a call is laid out: forms, shares and the parts of the workspace.
struct PagedLayout {
    int own_rb, pre_rb;        // row blocks of the two passes
    int own_slots, pre_slots;  // shares a kv head
    int max_tiles, n_records;
    bool by_tile;
    size_t records, own_slot_o, own_slot_lse, own_row_o, own_row_lse, pre_slot_o, pre_slot_lse,
        pre_row_o, pre_row_lse, bytes;
};

// Shares a CU, each with so many bytes of tables.  8-bit: as many as share it, or
// a whole number of times as many as its LDS holds at once: of more, all of one length,
// the rest would start when the others end.  us with four a CU and with the three that
// fit (32 heads over 8, d = 64): 100 requests of four tokens and 2000 keys 85 and 62, of
// 200 keys 25 and 28, 400 of 200 keys 81 and 59, 480 single tokens of 2000 keys 270 and
// 200.  At d = 128 two shares a CU stay where one workgroup fits, one after the other
// (which evens out calls that mix pieces and single tokens: 1023 of these beside 3070
// tokens behind 30000 keys, 32 heads over 4, 8.1 ms, with one share a CU 9.3).
template <typename S>
int shares_of(bool q8, int64_t tables)
{
    constexpr int64_t kLds = 160 * 1024, kGranule = 1280;  // of a CU, and of an allocation
    const int64_t each = (S::FIXED_LDS + tables + kGranule - 1) / kGranule * kGranule;
    const int fit = (int)std::max<int64_t>(1, std::min<int64_t>(S::WGS_PER_CU, kLds / each));
    return q8 ? S::WGS_PER_CU / fit * fit : S::WGS_PER_CU;
}
template <bool Q8>
int shares_per_cu(int rb, int d, int64_t tables)
{
    if (Q8 && rb == 8)
        return shares_of<PagedShape<128, 8, true>>(Q8, tables);
    if (Q8 && rb == 0)
        return d == 128 ? shares_of<PagedShape<128, 0, true>>(Q8, tables)
                        : shares_of<PagedShape<64, 0, true>>(Q8, tables);
    if (d == 128)
        return rb == 4 ? shares_of<PagedShape<128, 4, Q8>>(Q8, tables)
                       : shares_of<PagedShape<128, 1, Q8>>(Q8, tables);
    return rb == 4 ? shares_of<PagedShape<64, 4, Q8>>(Q8, tables)
                   : shares_of<PagedShape<64, 1, Q8>>(Q8, tables);
}

// LDS of the own-keys pass's tables.
int64_t table_bytes(int64_t max_tiles, int64_t batch, bool ragged)
{
    return 4 * (max_tiles + 1 + batch + (ragged ? 2 * (batch + 1) : 0));
}

// Rows of a tile.
int form_rows(int rb) { return rb == 0 ? 16 : 32 * rb; }

PagedLayout paged_layout(int32_t batch, int64_t total_tokens, bool ragged, bool prefix, int32_t hq,
                         int32_t hkv, int32_t d, bool q8)
{
    auto per_cu = [&](int rb, int64_t tables) {
        return q8 ? shares_per_cu<true>(rb, d, tables) : shares_per_cu<false>(rb, d, tables);
    };
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
    if (q8) {
        // 8-bit: tiles of 16 rows for single tokens (us with 32 and with 16: 96
        // requests of 64, of 955, of 3820 keys 19.6, 57, 152 and 16.2, 52, 148; a
        // request of more rows would read its keys more than once), and at d = 128
        // tiles of 256 for requests of more than 128 on average (us with 128 and with
        // 256: five requests of 40 tokens, of 256, of 500 to 1800 79, 241, 744 and 74,
        // 207, 620, the last with a cap 844 and 767; d = 64: 411 and 401, with a cap 587
        // and 625; the prefix's pass of 160 tokens, whose tiles are few, takes 5 more).
        // A call of unequal requests pays for the mean: 96 single tokens of 150 to 15000
        // keys (285 us) and a prompt of 3200 (161) 855 in tiles of 256, 1023 of 200 keys
        // (76) and 3070 tokens behind 30000 (1188; 32 heads over 4) 8078 in tiles of 32.
        if (!ragged || total_tokens <= batch)
            p.own_rb = 0;
        else if (d == 128 && total_tokens * group > (int64_t)batch * 128)
            p.own_rb = 8;
        if (total_tokens * group <= 16)
            p.pre_rb = 0;
    }
    const int64_t rows = form_rows(p.own_rb);
    p.max_tiles = (int)std::min<int64_t>(
        kMaxTiles + 1, ragged ? total_tokens * group / rows + batch : (int64_t)batch);
    const int64_t tables = table_bytes(p.max_tiles, batch, ragged);
    p.own_slots = std::max(1, kCus * per_cu(p.own_rb, tables) / hkv);
    p.pre_slots = std::max(1, kCus * per_cu(p.pre_rb, 0) / hkv);
    size_t at = 0;
    auto take = [&](size_t n) {
        const size_t here = at;
        at += (n + 255) / 256 * 256;
        return here;
    };
    // 8-bit: one a row tile where that is fewer, or where shares cut by charges too
    p.by_tile = prefix || (q8 && (p.own_rb <= 1 || p.max_tiles <= p.own_slots));
    p.n_records = p.by_tile ? p.max_tiles : p.own_slots;
    p.records = take((size_t)p.n_records * kRecordWords * 4);
    const size_t own = (size_t)2 * p.own_slots * hkv * rows;
    p.own_slot_o = take(own * d * 4);
    p.own_slot_lse = take(own * 4);
    if (prefix) {
        const size_t all = (size_t)total_tokens * hq;
        const size_t pre = (size_t)2 * p.pre_slots * hkv * form_rows(p.pre_rb);
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

template <int D, int RB, bool PREFIX, bool Q8>
void launch_scores(int score, dim3 grid, hipStream_t s, const PagedArgs &a)
{
    const dim3 threads(PagedShape<D, RB, Q8>::THREADS);
    const uint32_t lds = PREFIX ? 0 : (uint32_t)table_bytes(a.max_tiles, a.batch, a.cu_q);
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, threads, lds, s, a); };
    switch (score) {
    case 0: launch(paged_attn_kernel<D, RB, 0, PREFIX, Q8>); break;
    case 1: launch(paged_attn_kernel<D, RB, 1, PREFIX, Q8>); break;
    case 2: launch(paged_attn_kernel<D, RB, 2, PREFIX, Q8>); break;
    default: launch(paged_attn_kernel<D, RB, 3, PREFIX, Q8>); break;
    }
}

template <bool PREFIX, bool Q8>
hipError_t launch_pass(int d, int rb, int score, hipStream_t s, const PagedArgs &a)
{
    const dim3 grid((uint32_t)(a.slots * a.hkv));
    if constexpr (Q8 && !PREFIX)
        if (rb == 8) {
            launch_scores<128, 8, PREFIX, Q8>(score, grid, s, a);
            return hipGetLastError();
        }
    if constexpr (Q8)
        if (rb == 0) {
            if (d == 128)
                launch_scores<128, 0, PREFIX, Q8>(score, grid, s, a);
            else
                launch_scores<64, 0, PREFIX, Q8>(score, grid, s, a);
            return hipGetLastError();
        }
    if (d == 128 && rb == 1)
        launch_scores<128, 1, PREFIX, Q8>(score, grid, s, a);
    else if (d == 128)
        launch_scores<128, 4, PREFIX, Q8>(score, grid, s, a);
    else if (rb == 1)
        launch_scores<64, 1, PREFIX, Q8>(score, grid, s, a);
    else
        launch_scores<64, 4, PREFIX, Q8>(score, grid, s, a);
    return hipGetLastError();
}

size_t workspace_bytes_of(int32_t batch, int64_t total_tokens, int32_t ragged, int32_t prefix,
                          int32_t hq, int32_t hkv, int32_t head_dim, bool q8)
{
    if (batch < 0 || total_tokens < 0 || total_tokens > INT32_MAX || hq <= 0 || hkv <= 0 ||
        hq % hkv != 0 || hq / hkv > 8 || (head_dim != 64 && head_dim != 128))
        return 0;
    return paged_layout(batch, total_tokens, ragged != 0, prefix != 0, hq, hkv, head_dim, q8)
        .bytes;
}

// A call on either form of the cache (k_scale, v_scale: of the 8-bit one).
ta_status paged_attn(const char *fn, bool q8, const void *q, const void *k_cache,
                     const void *k_scale, const void *v_cache, const void *v_scale, void *o,
                     int32_t o_dtype, float *lse, const int32_t *kv_lens, const int32_t *cu_q,
                     const int32_t *block_table, int32_t batch, int32_t table_width,
                     const int32_t *prefix_pages, int32_t prefix_len, int64_t total_tokens,
                     int32_t hq, int32_t hkv, int32_t head_dim, int64_t num_pages,
                     int32_t page_size, float softmax_scale, float softcap, const float *slopes,
                     void *workspace, size_t workspace_bytes, void *stream)
{
    clear_error();
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
    const PagedLayout p = paged_layout(batch, total_tokens, cu_q != nullptr, prefix_len > 0, hq,
                                       hkv, head_dim, q8);
    const int64_t group = hq / hkv;
    if (p.max_tiles > kMaxTiles)
        return fail(TA_ERR_UNSUPPORTED, "%s: more than %d row tiles a kv head (pass fewer query "
                    "tokens at a time)", fn, kMaxTiles);
    // steps are counted in 32 bits
    const int64_t steps = (int64_t)p.max_tiles * ((int64_t)table_width * page_size / 64 + 1);
    const int pre_rows = form_rows(p.pre_rb);
    const int64_t pre_tiles = (total_tokens * group + pre_rows - 1) / pre_rows;
    if (steps > INT32_MAX / 2 || pre_tiles * (prefix_len / 64 + 1) > INT32_MAX / 2)
        return fail(TA_ERR_UNSUPPORTED, "%s: too many steps", fn);
    // the join: workgroups of a row tile, rows of each
    const int join_rows = cu_q ? form_rows(p.own_rb) : (int)group;
    // 8-bit: as many ways as a row has partials on average, at most
    int ways = 1;
    while (q8 && ways < kJoinThreads / 16 && 2 * ways * p.max_tiles <= p.own_slots)
        ways *= 2;
    const int chunk_rows = std::min(join_rows, kJoinThreads / 16 / ways);
    const int chunks = (join_rows + chunk_rows - 1) / chunk_rows;
    const int64_t wgs = std::max<int64_t>({p.own_slots, prefix_len > 0 ? p.pre_slots : 0,
                                           (int64_t)p.n_records * chunks}) * hkv;
    const int threads = p.own_rb == 8 ? PagedShape<128, 8, true>::THREADS : kJoinThreads;
    if (wgs * threads > UINT32_MAX)  // of a launch
        return fail(TA_ERR_UNSUPPORTED, "%s: grid too large", fn);
    if (total_tokens == 0 || batch == 0)
        return TA_OK;
    if (!q || !o || !kv_lens || (num_pages > 0 && (!k_cache || !v_cache)) ||
        (q8 && num_pages > 0 && (!k_scale || !v_scale)) ||
        (table_width > 0 && !block_table) || (prefix_len > 0 && !prefix_pages))
        return fail(TA_ERR_INVALID_ARG, "%s: NULL argument", fn);
    if (num_pages == 0)
        return fail(TA_ERR_INVALID_ARG, "%s: a cache without pages", fn);
    if (((uintptr_t)q | (uintptr_t)k_cache | (uintptr_t)v_cache | (uintptr_t)o) & 15)
        return fail(TA_ERR_INVALID_ARG, "%s: q, o and the caches must be 16-byte aligned", fn);
    if (((uintptr_t)k_scale | (uintptr_t)v_scale) & 3)
        return fail(TA_ERR_INVALID_ARG, "%s: the scales must be 4-byte aligned", fn);
    if (!workspace || workspace_bytes < p.bytes)
        return fail(TA_ERR_WORKSPACE, "%s: workspace of %zu bytes, need %zu", fn,
                    workspace ? workspace_bytes : (size_t)0, p.bytes);
    if ((uintptr_t)workspace & 15)
        return fail(TA_ERR_WORKSPACE, "%s: workspace must be 16-byte aligned", fn);
    {
        const int64_t rows = total_tokens * hq, held = (num_pages * hkv) << lp;
        const int64_t cache = held * head_dim * (q8 ? 1 : 2);
        const Span spans[] = {{o, rows * head_dim * (o_dtype == TA_OUT_F32 ? 4 : 2)},
                              {lse, 4 * rows},
                              {workspace, (int64_t)p.bytes},
                              {q, rows * head_dim * 2},
                              {k_cache, cache},
                              {v_cache, cache},
                              {k_scale, held},
                              {v_scale, held},
                              {kv_lens, 4LL * batch},
                              {cu_q, 4LL * batch + 4},
                              {block_table, 4LL * batch * table_width},
                              {prefix_len > 0 ? prefix_pages : nullptr,
                               4 * (((int64_t)prefix_len + page_size - 1) >> lp)},
                              {slopes, 4LL * hq}};
        if (spans_overlap(spans, 3, 13))
            return fail(TA_ERR_INVALID_ARG, "%s: an output overlaps another argument", fn);
    }
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    auto part = [&](size_t off) { return reinterpret_cast<float *>(ws + off); };
    PagedArgs a{};
    a.q = static_cast<const uint16_t *>(q);
    a.kc = static_cast<const unsigned char *>(k_cache);
    a.vc = static_cast<const unsigned char *>(v_cache);
    a.ks = static_cast<const unsigned char *>(k_scale);
    a.vs = static_cast<const unsigned char *>(v_scale);
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
    a.by_tile = p.by_tile;
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
        err = q8 ? launch_pass<true, true>(head_dim, p.pre_rb, score, s, b)
                 : launch_pass<true, false>(head_dim, p.pre_rb, score, s, b);
    }
    if (err == hipSuccess)
        err = q8 ? launch_pass<false, true>(head_dim, p.own_rb, score, s, a)
                 : launch_pass<false, false>(head_dim, p.own_rb, score, s, a);
    if (err == hipSuccess) {
        JoinArgs j{};
        j.o = o;
        j.lse = lse;
        j.records = a.records;
        j.slot_o = a.slot_o;
        j.slot_lse = a.slot_lse;
        j.tile_rows = form_rows(p.own_rb);
        j.charge = q8 && p.own_rb <= 1 ? PagedShape<128, 1, true>::CHARGE : 0;
        j.chunk_rows = chunk_rows;
        j.ways = ways;
        j.chunks = chunks;
        j.row_o = a.row_o;
        j.row_lse = a.row_lse;
        j.pre_slot_o = part(p.pre_slot_o);
        j.pre_slot_lse = part(p.pre_slot_lse);
        j.pre_row_o = part(p.pre_row_o);
        j.pre_row_lse = part(p.pre_row_lse);
        j.prefix_len = prefix_len;
        j.pre_rows = pre_rows;
        // (steps are as long for either head_dim)
        const int step = p.pre_rb == 4 ? PagedShape<128, 4, false>::STEP
                         : q8          ? PagedShape<128, 1, true>::STEP
                                       : PagedShape<128, 1, false>::STEP;
        j.pre_steps = (prefix_len + step - 1) / step;
        j.pre_share =
            (int32_t)std::max<int64_t>(p.pre_rb != 4 ? PagedShape<128, 1, false>::LEAST
                                       : q8          ? PagedShape<128, 4, true>::LEAST
                                                     : PagedShape<128, 4, false>::LEAST,
                                       (pre_tiles * j.pre_steps + p.pre_slots - 1) / p.pre_slots);
        j.slopes = slopes;
        j.total_tokens = (int32_t)total_tokens;
        j.hq = hq;
        j.hkv = hkv;
        j.group = (int32_t)group;
        j.o_f32 = a.o_f32;
        const dim3 grid((uint32_t)(p.n_records * chunks * hkv));
        const auto join =
            head_dim == 128
                ? (ways > 1 ? paged_join_kernel<128, true> : paged_join_kernel<128, false>)
                : (ways > 1 ? paged_join_kernel<64, true> : paged_join_kernel<64, false>);
        hipLaunchKernelGGL(join, grid, dim3(kJoinThreads), 0, s, j);
        err = hipGetLastError();
    }
    if (err != hipSuccess)
        return fail(TA_ERR_HIP, "%s: %s", fn, hipGetErrorString(err));
    return TA_OK;
}

}  // namespace
}  // namespace triattn

using namespace triattn;

extern "C" size_t ta_paged_workspace_bytes(int32_t batch, int64_t total_tokens, int32_t ragged,
                                           int32_t prefix, int32_t hq, int32_t hkv,
                                           int32_t head_dim)
{
    return workspace_bytes_of(batch, total_tokens, ragged, prefix, hq, hkv, head_dim, false);
}

extern "C" size_t ta_paged_q8_workspace_bytes(int32_t batch, int64_t total_tokens, int32_t ragged,
                                              int32_t prefix, int32_t hq, int32_t hkv,
                                              int32_t head_dim)
{
    return workspace_bytes_of(batch, total_tokens, ragged, prefix, hq, hkv, head_dim, true);
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
    return paged_attn("paged_attn_fwd", false, q, k_cache, nullptr, v_cache, nullptr, o, o_dtype,
                      lse, kv_lens, cu_q, block_table, batch, table_width, prefix_pages, prefix_len,
                      total_tokens, hq, hkv, head_dim, num_pages, page_size, softmax_scale,
                      softcap, slopes, workspace, workspace_bytes, stream);
}

extern "C" ta_status paged_attn_fwd_q8(
    const void *q, const void *k_cache, const void *k_scale, const void *v_cache,
    const void *v_scale, void *o, int32_t o_dtype, float *lse, const int32_t *kv_lens,
    const int32_t *cu_q, const int32_t *block_table, int32_t batch, int32_t table_width,
    const int32_t *prefix_pages, int32_t prefix_len, int64_t total_tokens, int32_t hq, int32_t hkv,
    int32_t head_dim, int64_t num_pages, int32_t page_size, float softmax_scale, float softcap,
    const float *slopes, void *workspace, size_t workspace_bytes, void *stream)
{
    return paged_attn("paged_attn_fwd_q8", true, q, k_cache, k_scale, v_cache, v_scale, o, o_dtype,
                      lse, kv_lens, cu_q, block_table, batch, table_width, prefix_pages, prefix_len,
                      total_tokens, hq, hkv, head_dim, num_pages, page_size, softmax_scale,
                      softcap, slopes, workspace, workspace_bytes, stream);
}
