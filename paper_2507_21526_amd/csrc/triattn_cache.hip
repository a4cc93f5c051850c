// The paged K/V cache of libtriattn.so: page maps of a serving step, and the
// rows of new tokens written into their pages.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "triattn_device.h"
#include "triattn_internal.h"
#include "triattn_spans.h"

namespace triattn {
namespace {

constexpr int kMapThreads = 256;
constexpr int kMapSlots = 1024;  // slots of a workgroup
constexpr int kMapPer = TA_MAX_BATCH / kMapThreads;  // requests of a thread

struct MapArgs {
    const int32_t *cached;
    const int32_t *fresh;
    int32_t *table;
    const int32_t *free_pages;
    const int32_t *n_free;
    int32_t *kv_lens;
    int32_t *cu_new;
    int32_t *slots;
    int32_t *state;
    int64_t slot_count;
    int32_t batch, width, free_capacity, page_log2;
};

// Exclusive scan of one value a thread over the workgroup (and the total).
__device__ __forceinline__ int64_t map_scan(int64_t x, int64_t *wave_sum, int64_t &total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t inc = x;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int64_t y = __shfl_up(inc, o);
        inc += lane >= o ? y : 0;
    }
    if (lane == 63)
        wave_sum[wave] = inc;
    __syncthreads();
    int64_t base = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kMapThreads / 64; ++w) {
        base += w < wave ? wave_sum[w] : 0;
        total += wave_sum[w];
    }
    __syncthreads();
    return base + inc - x;
}

// Pages and slots of one step, all or nothing.  Every workgroup scans the
// requests for itself (a few KB that stay in L2), so that one launch does:
// no workgroup waits for another, and whether the step fits is the same
// everywhere.  A workgroup then finds the request of each of its slots by
// binary search.  The token that opens a page writes its table entry; a token
// in a page that was there before reads the entry, which nothing writes.
__global__ __launch_bounds__(kMapThreads) void page_map_kernel(MapArgs a)
{
    __shared__ int32_t s_cu[TA_MAX_BATCH + 1];    // first new token
    __shared__ int32_t s_page[TA_MAX_BATCH];      // rank of the first new page
    __shared__ int32_t s_cached[TA_MAX_BATCH];
    __shared__ int64_t s_wave[kMapThreads / 64];
    __shared__ int32_t s_bad;
    const int tid = threadIdx.x;
    const int64_t page = (int64_t)1 << a.page_log2;
    const int per = (a.batch + kMapThreads - 1) / kMapThreads;
    const int32_t n_free = a.n_free[0];
    if (tid == 0)
        s_bad = 0;
    int32_t c[kMapPer], f[kMapPer];
    int64_t toks = 0, need = 0;
    int bad = n_free < 0 || n_free > a.free_capacity ? TA_MAP_BAD_FREE : 0;
#pragma unroll
    for (int i = 0; i < kMapPer; ++i) {
        const int b = tid * per + i;
        const bool on = i < per && b < a.batch;
        c[i] = on ? a.cached[b] : 0;
        f[i] = on ? a.fresh[b] : 0;
        if ((c[i] < 0) | (f[i] < 0)) {
            bad |= TA_MAP_BAD_LENGTH;
            c[i] = f[i] = 0;
        }
        const int64_t old_pages = (c[i] + page - 1) >> a.page_log2;
        const int64_t all_pages = ((int64_t)c[i] + f[i] + page - 1) >> a.page_log2;
        if (all_pages > a.width)
            bad |= TA_MAP_TABLE_WIDTH;
        toks += f[i];
        need += all_pages - old_pages;
    }
    int64_t n_toks, n_need;
    int64_t t = map_scan(toks, s_wave, n_toks);
    int64_t p = map_scan(need, s_wave, n_need);
    if (n_need > n_free)
        bad |= TA_MAP_NO_PAGES;
    if (n_toks > a.slot_count)
        bad |= TA_MAP_SLOT_COUNT;
    if (bad)
        atomicOr(&s_bad, bad);
    // (totals past 32 bits are refused above: slot_count and n_free are not)
#pragma unroll
    for (int i = 0; i < kMapPer; ++i) {
        const int b = tid * per + i;
        if (i < per && b < a.batch) {
            s_cu[b] = (int32_t)t;
            s_page[b] = (int32_t)p;
            s_cached[b] = c[i];
            t += f[i];
            p += (((int64_t)c[i] + f[i] + page - 1) >> a.page_log2) -
                 ((c[i] + page - 1) >> a.page_log2);
        }
    }
    if (tid == 0)
        s_cu[a.batch] = (int32_t)n_toks;
    __syncthreads();
    bad = s_bad;
    if (blockIdx.x == 0) {
        for (int b = tid; b <= a.batch; b += kMapThreads) {
            a.cu_new[b] = bad ? 0 : s_cu[b];
            if (b < a.batch)
                a.kv_lens[b] = bad ? a.cached[b] : s_cached[b] + s_cu[b + 1] - s_cu[b];
        }
        if (tid == 0) {
            a.state[0] = bad ? n_free : (int32_t)(n_free - n_need);
            a.state[1] = bad;
        }
    }
    const int64_t first = (int64_t)blockIdx.x * kMapSlots;
    for (int64_t i = first + tid; i < min(first + kMapSlots, a.slot_count); i += kMapThreads) {
        if (bad || i >= n_toks) {
            a.slots[i] = -1;
            continue;
        }
        // the request with cu[b] <= i < cu[b + 1]
        int lo = 0, hi = a.batch;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (s_cu[mid] <= i)
                lo = mid;
            else
                hi = mid;
        }
        const int32_t had = s_cached[lo];
        const int32_t pos = had + (int32_t)(i - s_cu[lo]);
        const int32_t x = pos >> a.page_log2, in = pos & (int32_t)(page - 1);
        const int32_t old_pages = (int32_t)((had + page - 1) >> a.page_log2);
        int32_t *entry = a.table + (int64_t)lo * a.width + x;
        int32_t id;
        if (x < old_pages) {
            id = *entry;
        } else {
            id = a.free_pages[n_free - 1 - (s_page[lo] + x - old_pages)];
            if (in == 0)
                *entry = id;
        }
        // an entry that is no page gives no slot
        const int64_t slot = ((int64_t)id << a.page_log2) + in;
        a.slots[i] = id < 0 || slot > INT32_MAX ? -1 : (int32_t)slot;
    }
}

struct WriteArgs {
    const uint16_t *k, *v;
    uint16_t *kc, *vc;
    const int32_t *slots;
    int64_t k_token, k_head, v_token, v_head;  // strides in elements
    int64_t total_tokens, n_slots;
    int32_t hkv, page_log2;
    uint32_t rows;  // (token, head) rows of a workgroup
};

// One 16-byte chunk of K and of V a thread and turn.
template <int D>
__global__ __launch_bounds__(256) void cache_write_kernel(WriteArgs a)
{
    constexpr int CHUNKS = D / 8;
    const int64_t total = a.total_tokens * a.hkv;
    const int64_t r0 = (int64_t)blockIdx.x * a.rows;
    const int chunk = threadIdx.x % CHUNKS;
    for (uint32_t i = threadIdx.x / CHUNKS; i < a.rows; i += 256 / CHUNKS) {
        const int64_t r = r0 + i;
        if (r >= total)
            return;
        const int64_t tok = r / a.hkv;
        const int head = (int)(r - tok * a.hkv);
        const int64_t slot = a.slots[tok];
        if (slot < 0 || slot >= a.n_slots)
            continue;
        const u32x4 kk =
            *reinterpret_cast<const u32x4 *>(a.k + tok * a.k_token + head * a.k_head + chunk * 8);
        const u32x4 vv =
            *reinterpret_cast<const u32x4 *>(a.v + tok * a.v_token + head * a.v_head + chunk * 8);
        const int64_t to =
            (((((slot >> a.page_log2) * a.hkv + head) << a.page_log2) +
              (slot & (((int64_t)1 << a.page_log2) - 1))) *
             D) +
            chunk * 8;
        *reinterpret_cast<u32x4 *>(a.kc + to) = kk;
        *reinterpret_cast<u32x4 *>(a.vc + to) = vv;
    }
}

}  // namespace

int page_log2(int32_t page_size)
{
    for (int l = 4; l <= 8; ++l)
        if (page_size == 1 << l)
            return l;
    return -1;
}

}  // namespace triattn

using namespace triattn;

extern "C" ta_status ta_page_map(const int32_t *cached_lens, const int32_t *new_lens,
                                 int32_t batch, int32_t page_size, int32_t *block_table,
                                 int32_t table_width, const int32_t *free_pages,
                                 int32_t free_capacity, const int32_t *n_free, int32_t *kv_lens,
                                 int32_t *cu_new, int32_t *slots, int64_t slot_count,
                                 int32_t *state, void *stream)
{
    clear_error();
    const char *fn = "ta_page_map";
    if (batch < 0 || table_width < 0 || free_capacity < 0 || slot_count < 0)
        return fail(TA_ERR_INVALID_ARG, "%s: negative size", fn);
    if (batch > TA_MAX_BATCH)
        return fail(TA_ERR_UNSUPPORTED, "%s: batch %d > %d", fn, batch, TA_MAX_BATCH);
    const int lp = page_log2(page_size);
    if (lp < 0)
        return fail(TA_ERR_UNSUPPORTED, "%s: page_size %d not in {16, 32, 64, 128, 256}", fn,
                    page_size);
    if ((int64_t)table_width * page_size > INT32_MAX || slot_count > INT32_MAX)
        return fail(TA_ERR_UNSUPPORTED, "%s: positions or slots past 32 bits", fn);
    if (!n_free || !cu_new || !state ||
        (batch > 0 && (!cached_lens || !new_lens || !kv_lens)) ||
        (batch > 0 && table_width > 0 && !block_table) || (free_capacity > 0 && !free_pages) ||
        (slot_count > 0 && !slots))
        return fail(TA_ERR_INVALID_ARG, "%s: NULL argument", fn);
    // Workgroups read the inputs at any time: no output may lie on one, nor
    // on another output.
    const Span spans[] = {{kv_lens, 4LL * batch},
                          {cu_new, 4LL * batch + 4},
                          {slots, 4 * slot_count},
                          {state, 8},
                          {block_table, 4LL * batch * table_width},
                          {cached_lens, 4LL * batch},
                          {new_lens, 4LL * batch},
                          {free_pages, 4LL * free_capacity},
                          {n_free, 4}};
    if (spans_overlap(spans, 5, 9))
        return fail(TA_ERR_INVALID_ARG, "%s: an output overlaps another argument", fn);
    MapArgs a{};
    a.cached = cached_lens;
    a.fresh = new_lens;
    a.table = block_table;
    a.free_pages = free_pages;
    a.n_free = n_free;
    a.kv_lens = kv_lens;
    a.cu_new = cu_new;
    a.slots = slots;
    a.state = state;
    a.slot_count = slot_count;
    a.batch = batch;
    a.width = table_width;
    a.free_capacity = free_capacity;
    a.page_log2 = lp;
    const int64_t wgs = std::max<int64_t>(1, (slot_count + kMapSlots - 1) / kMapSlots);
    hipLaunchKernelGGL(page_map_kernel, dim3((uint32_t)wgs), dim3(kMapThreads), 0,
                       static_cast<hipStream_t>(stream), a);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess)
        return fail(TA_ERR_HIP, "%s: %s", fn, hipGetErrorString(err));
    return TA_OK;
}

extern "C" ta_status kv_cache_write(const void *k, const void *v, int64_t k_token_stride,
                                    int64_t k_head_stride, int64_t v_token_stride,
                                    int64_t v_head_stride, const int32_t *slots,
                                    int64_t total_tokens, void *k_cache, void *v_cache,
                                    int64_t num_pages, int32_t hkv, int32_t page_size,
                                    int32_t head_dim, void *stream)
{
    clear_error();
    const char *fn = "kv_cache_write";
    if (total_tokens < 0 || num_pages < 0 || hkv <= 0)
        return fail(TA_ERR_INVALID_ARG, "%s: negative size or no heads", fn);
    if (head_dim != 64 && head_dim != 128)
        return fail(TA_ERR_UNSUPPORTED, "%s: head_dim %d not in {64, 128}", fn, head_dim);
    const int lp = page_log2(page_size);
    if (lp < 0)
        return fail(TA_ERR_UNSUPPORTED, "%s: page_size %d not in {16, 32, 64, 128, 256}", fn,
                    page_size);
    if (num_pages > INT32_MAX / page_size)
        return fail(TA_ERR_UNSUPPORTED, "%s: slots past 32 bits", fn);
    if (total_tokens == 0 || num_pages == 0)
        return TA_OK;
    if (!k || !v || !slots || !k_cache || !v_cache)
        return fail(TA_ERR_INVALID_ARG, "%s: NULL argument", fn);
    if (((uintptr_t)k | (uintptr_t)v | (uintptr_t)k_cache | (uintptr_t)v_cache) & 15)
        return fail(TA_ERR_INVALID_ARG, "%s: k, v and the caches must be 16-byte aligned", fn);
    if ((k_token_stride | k_head_stride | v_token_stride | v_head_stride) & 7)
        return fail(TA_ERR_INVALID_ARG, "%s: strides must be multiples of 8 elements", fn);
    if (k_token_stride < 0 || k_head_stride < 0 || v_token_stride < 0 || v_head_stride < 0)
        return fail(TA_ERR_INVALID_ARG, "%s: negative stride", fn);
    const int64_t cache = ((num_pages * hkv) << lp) * head_dim * 2;
    const Span spans[] = {
        {k_cache, cache},
        {v_cache, cache},
        {k, 2 * ((total_tokens - 1) * k_token_stride + (hkv - 1) * k_head_stride + head_dim)},
        {v, 2 * ((total_tokens - 1) * v_token_stride + (hkv - 1) * v_head_stride + head_dim)},
        {slots, 4 * total_tokens}};
    if (spans_overlap(spans, 2, 5))
        return fail(TA_ERR_INVALID_ARG, "%s: a cache overlaps another argument", fn);
    WriteArgs a{};
    a.k = static_cast<const uint16_t *>(k);
    a.v = static_cast<const uint16_t *>(v);
    a.kc = static_cast<uint16_t *>(k_cache);
    a.vc = static_cast<uint16_t *>(v_cache);
    a.slots = slots;
    a.k_token = k_token_stride;
    a.k_head = k_head_stride;
    a.v_token = v_token_stride;
    a.v_head = v_head_stride;
    a.total_tokens = total_tokens;
    a.n_slots = num_pages << lp;
    a.hkv = hkv;
    a.page_log2 = lp;
    // one row a thread group, more where a launch (2^32 threads at most) does
    // not hold that many
    constexpr int64_t kMaxWgs = 1 << 22;
    const int64_t rows = total_tokens * hkv, turn = 256 / (head_dim / 8);
    const int64_t turns = std::max<int64_t>(1, (rows + turn * kMaxWgs - 1) / (turn * kMaxWgs));
    if (turns * turn > INT32_MAX)
        return fail(TA_ERR_UNSUPPORTED, "%s: too many rows", fn);
    a.rows = (uint32_t)(turns * turn);
    const int64_t wgs = (rows + a.rows - 1) / a.rows;
    if (head_dim == 128)
        hipLaunchKernelGGL(cache_write_kernel<128>, dim3((uint32_t)wgs), dim3(256), 0,
                           static_cast<hipStream_t>(stream), a);
    else
        hipLaunchKernelGGL(cache_write_kernel<64>, dim3((uint32_t)wgs), dim3(256), 0,
                           static_cast<hipStream_t>(stream), a);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess)
        return fail(TA_ERR_HIP, "%s: %s", fn, hipGetErrorString(err));
    return TA_OK;
}
