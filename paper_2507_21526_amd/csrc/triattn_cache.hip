// The paged K/V cache of libtriattn.so: page maps of a serving step, the rows of
// new tokens written into their pages, as they are or quantised to 8 bits, and
// cached rows read back.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <cstdlib>

#include "triattn_device.h"
#include "triattn_internal.h"
#include "triattn_rows8.h"
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
    void *kc, *vc;
    uint8_t *ks, *vs;  // scales of an 8-bit cache
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
        *reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(a.kc) + to) = kk;
        *reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(a.vc) + to) = vv;
    }
}

// a / b where both fit 32 bits, without the long division of 64-bit numbers.
__device__ __forceinline__ int64_t div_rows(int64_t a, int32_t b, bool small)
{
    return small ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}

// Eight bf16 values of a row, which LANES lanes hold, quantised: the scale's byte,
// and the elements in two words.  |x| as a bf16 number without its sign orders like
// an integer.  With the row's largest finite one, 2^(E - 127) (1 + M / 128), the
// least e with |x| <= 448 2^e = 1.75 2^(e + 8) is E - 135, one more where M > 96.
template <int LANES>
__device__ __forceinline__ uint32_t quantise8(u32x4 x, uint32_t (&out)[2])
{
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    constexpr uint32_t kInf = 0x7f80;
    u16x2 m2{};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        m2 = __builtin_elementwise_max(m2, __builtin_bit_cast(u16x2, x[i] & 0x7fff7fffu));
    uint32_t top = max(m2[0], m2[1]);
    bool odd = top >= kInf;  // infinite or NaN values: they set no scale
    if (odd) {
        top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t b = (x[i / 2] >> (16 * (i & 1))) & 0x7fff;
            top = max(top, b < kInf ? b : 0);
        }
    }
#pragma unroll
    for (int o = LANES / 2; o >= 1; o >>= 1)
        top = max(top, (uint32_t)__shfl_xor((int)top, o, LANES));
    const uint32_t byte = (uint32_t)max((int)(top >> 7) - 8 + ((top & 127) > 96 ? 1 : 0),
                                        kLeastExp + 127);
    const float inv = __uint_as_float((254 - byte) << 23);  // 2^-e
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
        f[i] = __uint_as_float(i & 1 ? x[i / 2] & 0xffff0000u : x[i / 2] << 16) * inv;
    if (byte == kMostExp + 127 || odd) {
        // 256 2^120 is past fp32 and bf16: 240 is as far as it goes there
        const float most = byte == kMostExp + 127 ? 240.f : 448.f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            f[i] = fabsf(f[i]) < INFINITY ? fminf(fmaxf(f[i], -most), most) : __builtin_nanf("");
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i], f[4 * i + 1], 0, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i + 2], f[4 * i + 3], w, true);
        out[i] = (uint32_t)w;
    }
    return byte;
}

// Quantises a row of K and one of V a group of D / 8 lanes and turn: 16 bytes read
// and 8 written a lane.
template <int D>
__global__ __launch_bounds__(256) void cache_write8_kernel(WriteArgs a)
{
    constexpr int LANES = D / 8;
    const int64_t total = a.total_tokens * a.hkv;
    const int64_t r0 = (int64_t)blockIdx.x * a.rows;
    const bool small = total <= UINT32_MAX;
    const int lane = threadIdx.x % LANES;
    for (uint32_t i = threadIdx.x / LANES; i < a.rows; i += 256 / LANES) {
        const int64_t r = r0 + i;
        if (r >= total)
            return;
        const int64_t tok = div_rows(r, a.hkv, small);
        const int head = (int)(r - tok * a.hkv);
        const int64_t slot = a.slots[tok];
        if (slot < 0 || slot >= a.n_slots)
            continue;
        const u32x4 kk =
            *reinterpret_cast<const u32x4 *>(a.k + tok * a.k_token + head * a.k_head + lane * 8);
        const u32x4 vv =
            *reinterpret_cast<const u32x4 *>(a.v + tok * a.v_token + head * a.v_head + lane * 8);
        const int64_t row = ((((slot >> a.page_log2) * a.hkv + head) << a.page_log2) +
                             (slot & (((int64_t)1 << a.page_log2) - 1)));
        uint32_t ko[2], vo[2];
        const uint32_t kb = quantise8<LANES>(kk, ko), vb = quantise8<LANES>(vv, vo);
        *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(a.kc) + row * D + lane * 8) =
            make_uint2(ko[0], ko[1]);
        *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(a.vc) + row * D + lane * 8) =
            make_uint2(vo[0], vo[1]);
        if (lane == 0) {
            a.ks[row] = (uint8_t)kb;
            a.vs[row] = (uint8_t)vb;
        }
    }
}

constexpr int kReadTokens = 16;  // of a workgroup

struct ReadArgs {
    const void *kc, *vc;
    const uint8_t *ks, *vs;
    const int32_t *table, *cu, *starts;
    uint16_t *k, *v;
    int64_t k_token, k_head, v_token, v_head;  // strides in elements
    int64_t total_tokens;
    int32_t blocks;  // of kReadTokens tokens
    int32_t batch, width, hkv, page_log2, num_pages;
};

// Rows of the cache as bf16, D / 8 lanes a row: 16 bytes written a lane, and 8
// (16: bf16) read.  Every workgroup checks the offsets for itself and finds the
// places of its tokens by binary search.
template <int D, bool Q8>
__global__ __launch_bounds__(256) void cache_read_kernel(ReadArgs a)
{
    constexpr int LANES = D / 8;
    __shared__ int32_t s_cu[TA_MAX_BATCH + 1];
    __shared__ int32_t s_slot[kReadTokens];  // -1: no page, -2: past the last request
    const int tid = threadIdx.x;
    bool bad = false;
    for (int b = tid; b <= a.batch; b += 256) {
        const int32_t x = a.cu[b];
        s_cu[b] = x;
        bad |= b == 0 ? x != 0 : x < a.cu[b - 1];
        bad |= x > a.total_tokens;
    }
    bad = __syncthreads_or(bad);
    const int lane = tid % LANES;
    const uint32_t rows = (uint32_t)kReadTokens * (uint32_t)a.hkv;
    for (int32_t block = blockIdx.x; block < a.blocks; block += gridDim.x) {
        const int64_t first = (int64_t)block * kReadTokens;
        if (tid < kReadTokens) {
            const int64_t tok = first + tid;
            int32_t slot = -1;
            if (!bad) {
                slot = -2;
                if (tok < s_cu[a.batch]) {
                    int lo = 0, hi = a.batch;
                    while (hi - lo > 1) {
                        const int mid = (lo + hi) >> 1;
                        if (s_cu[mid] <= tok)
                            lo = mid;
                        else
                            hi = mid;
                    }
                    const int64_t pos = tok - s_cu[lo] + (a.starts ? a.starts[lo] : 0);
                    const int64_t page = pos >> a.page_log2;
                    int32_t id = -1;
                    if (pos >= 0 && page < a.width)
                        id = a.table[(int64_t)lo * a.width + page];
                    slot = id < 0 || id >= a.num_pages
                               ? -1
                               : (id << a.page_log2) + (int32_t)(pos & ((1 << a.page_log2) - 1));
                }
            }
            s_slot[tid] = tok < a.total_tokens ? slot : -2;
        }
        __syncthreads();
        for (uint32_t r = tid / LANES; r < rows; r += 256 / LANES) {
            const uint32_t t = r / (uint32_t)a.hkv, head = r - t * (uint32_t)a.hkv;
            const int32_t slot = s_slot[t];
            if (slot == -2)
                continue;
            const int64_t tok = first + t;
            u32x4 out[2];
            if (slot < 0) {
                out[0] = out[1] = u32x4{0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u};
            } else {
                const int64_t row =
                    (((int64_t)(slot >> a.page_log2) * a.hkv + head) << a.page_log2) +
                    (slot & ((1 << a.page_log2) - 1));
                const int64_t at = row * D + lane * 8;
                if constexpr (Q8) {
                    const uint2 kk =
                        *reinterpret_cast<const uint2 *>(static_cast<const uint8_t *>(a.kc) + at);
                    const uint2 vv =
                        *reinterpret_cast<const uint2 *>(static_cast<const uint8_t *>(a.vc) + at);
                    const float kf = q8_scale_bits(a.ks[row]), vf = q8_scale_bits(a.vs[row]);
                    out[0] = __builtin_bit_cast(u32x4, q8_fragment(kk.x, kk.y, kf));
                    out[1] = __builtin_bit_cast(u32x4, q8_fragment(vv.x, vv.y, vf));
                } else {
                    out[0] =
                        *reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(a.kc) + at);
                    out[1] =
                        *reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(a.vc) + at);
                }
            }
            *reinterpret_cast<u32x4 *>(a.k + tok * a.k_token + head * a.k_head + lane * 8) = out[0];
            *reinterpret_cast<u32x4 *>(a.v + tok * a.v_token + head * a.v_head + lane * 8) = out[1];
        }
        __syncthreads();  // the places are read
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

// Both forms of the cache (k_scale, v_scale: of the 8-bit one).
static ta_status cache_write(const char *fn, bool q8, const void *k, const void *v,
                             int64_t k_token_stride, int64_t k_head_stride,
                             int64_t v_token_stride, int64_t v_head_stride, const int32_t *slots,
                             int64_t total_tokens, void *k_cache, void *k_scale, void *v_cache,
                             void *v_scale, int64_t num_pages, int32_t hkv, int32_t page_size,
                             int32_t head_dim, void *stream)
{
    clear_error();
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
    if (!k || !v || !slots || !k_cache || !v_cache || (q8 && (!k_scale || !v_scale)))
        return fail(TA_ERR_INVALID_ARG, "%s: NULL argument", fn);
    if (((uintptr_t)k | (uintptr_t)v | (uintptr_t)k_cache | (uintptr_t)v_cache) & 15)
        return fail(TA_ERR_INVALID_ARG, "%s: k, v and the caches must be 16-byte aligned", fn);
    if ((k_token_stride | k_head_stride | v_token_stride | v_head_stride) & 7)
        return fail(TA_ERR_INVALID_ARG, "%s: strides must be multiples of 8 elements", fn);
    if (k_token_stride < 0 || k_head_stride < 0 || v_token_stride < 0 || v_head_stride < 0)
        return fail(TA_ERR_INVALID_ARG, "%s: negative stride", fn);
    const int64_t held = (num_pages * hkv) << lp, cache = held * head_dim * (q8 ? 1 : 2);
    const Span spans[] = {
        {k_cache, cache},
        {v_cache, cache},
        {k_scale, held},
        {v_scale, held},
        {k, 2 * ((total_tokens - 1) * k_token_stride + (hkv - 1) * k_head_stride + head_dim)},
        {v, 2 * ((total_tokens - 1) * v_token_stride + (hkv - 1) * v_head_stride + head_dim)},
        {slots, 4 * total_tokens}};
    if (spans_overlap(spans, 4, 7))
        return fail(TA_ERR_INVALID_ARG, "%s: a cache overlaps another argument", fn);
    WriteArgs a{};
    a.k = static_cast<const uint16_t *>(k);
    a.v = static_cast<const uint16_t *>(v);
    a.kc = k_cache;
    a.vc = v_cache;
    a.ks = static_cast<uint8_t *>(k_scale);
    a.vs = static_cast<uint8_t *>(v_scale);
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
    const auto kernel = q8 ? (head_dim == 128 ? cache_write8_kernel<128> : cache_write8_kernel<64>)
                           : (head_dim == 128 ? cache_write_kernel<128> : cache_write_kernel<64>);
    hipLaunchKernelGGL(kernel, dim3((uint32_t)wgs), dim3(256), 0, static_cast<hipStream_t>(stream),
                       a);
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
    return cache_write("kv_cache_write", false, k, v, k_token_stride, k_head_stride,
                       v_token_stride, v_head_stride, slots, total_tokens, k_cache, nullptr,
                       v_cache, nullptr, num_pages, hkv, page_size, head_dim, stream);
}

extern "C" ta_status kv_cache_write_q8(const void *k, const void *v, int64_t k_token_stride,
                                       int64_t k_head_stride, int64_t v_token_stride,
                                       int64_t v_head_stride, const int32_t *slots,
                                       int64_t total_tokens, void *k_cache, void *k_scale,
                                       void *v_cache, void *v_scale, int64_t num_pages,
                                       int32_t hkv, int32_t page_size, int32_t head_dim,
                                       void *stream)
{
    return cache_write("kv_cache_write_q8", true, k, v, k_token_stride, k_head_stride,
                       v_token_stride, v_head_stride, slots, total_tokens, k_cache, k_scale,
                       v_cache, v_scale, num_pages, hkv, page_size, head_dim, stream);
}

namespace {

// The rows of an output [tokens, heads, d] of bf16 with its strides in elements.
struct RowSet {
    uintptr_t at;
    int64_t token, head;  // strides
    int64_t tokens, heads, d;

    int64_t extent() const { return (tokens - 1) * token + (heads - 1) * head + d; }

    // Whether no two rows share an element: the heads of a token lie within its
    // stride, or the tokens of a head within the head's.
    bool apart() const
    {
        if (tokens == 1)
            return heads == 1 || head >= d;
        if (heads == 1)
            return token >= d;
        return token >= head ? head >= d && (token - d) / head >= heads - 1
                             : token >= d && (head - d) / token >= tokens - 1;
    }

    // Whether a row may share an element with one of another output of the same
    // sizes: views that alternate in one buffer do not.
    bool meets(const RowSet &o) const
    {
        const uintptr_t lo = std::min(at, o.at), hi = std::max(at, o.at);
        const RowSet &first = at <= o.at ? *this : o;
        if (hi - lo >= (uintptr_t)(2 * first.extent()))
            return false;
        if ((tokens > 1 && token != o.token) || (heads > 1 && head != o.head))
            return true;
        for (int64_t j = 1 - heads; j < heads; ++j) {
            // two rows j heads apart, and some tokens: the nearest ones
            const int64_t x = (int64_t)((hi - lo) / 2) + (heads > 1 ? j * head : 0);
            const int64_t q = tokens > 1 ? x / token : 0;
            for (int64_t i = q - 1; i <= q + 1; ++i)
                if (std::abs(i) < tokens && std::abs(x - (tokens > 1 ? i * token : 0)) < d)
                    return true;
        }
        return false;
    }
};

}  // namespace

static ta_status cache_read(const char *fn, bool q8, const void *k_cache, const void *k_scale,
                            const void *v_cache, const void *v_scale, const int32_t *block_table,
                            int32_t batch, int32_t table_width, const int32_t *cu,
                            const int32_t *starts, void *k, void *v, int64_t k_token_stride,
                            int64_t k_head_stride, int64_t v_token_stride, int64_t v_head_stride,
                            int64_t total_tokens, int64_t num_pages, int32_t hkv,
                            int32_t page_size, int32_t head_dim, void *stream)
{
    clear_error();
    if (batch < 0 || table_width < 0 || total_tokens < 0 || num_pages < 0 || hkv <= 0)
        return fail(TA_ERR_INVALID_ARG, "%s: negative size or no heads", fn);
    if (batch > TA_MAX_BATCH)
        return fail(TA_ERR_UNSUPPORTED, "%s: batch %d > %d", fn, batch, TA_MAX_BATCH);
    if (head_dim != 64 && head_dim != 128)
        return fail(TA_ERR_UNSUPPORTED, "%s: head_dim %d not in {64, 128}", fn, head_dim);
    const int lp = page_log2(page_size);
    if (lp < 0)
        return fail(TA_ERR_UNSUPPORTED, "%s: page_size %d not in {16, 32, 64, 128, 256}", fn,
                    page_size);
    if (num_pages > INT32_MAX / page_size || (int64_t)table_width * page_size > INT32_MAX ||
        total_tokens > INT32_MAX || hkv > INT32_MAX / kReadTokens)
        return fail(TA_ERR_UNSUPPORTED, "%s: positions, slots or rows past 32 bits", fn);
    if (total_tokens == 0 || batch == 0)
        return TA_OK;
    if (!cu || !k || !v || (table_width > 0 && !block_table) ||
        (num_pages > 0 && (!k_cache || !v_cache || (q8 && (!k_scale || !v_scale)))))
        return fail(TA_ERR_INVALID_ARG, "%s: NULL argument", fn);
    if (((uintptr_t)k | (uintptr_t)v | (uintptr_t)k_cache | (uintptr_t)v_cache) & 15)
        return fail(TA_ERR_INVALID_ARG, "%s: k, v and the caches must be 16-byte aligned", fn);
    if ((k_token_stride | k_head_stride | v_token_stride | v_head_stride) & 7)
        return fail(TA_ERR_INVALID_ARG, "%s: strides must be multiples of 8 elements", fn);
    // rows that lie on one another would be written by several at once
    const RowSet ks{(uintptr_t)k, k_token_stride, k_head_stride, total_tokens, hkv, head_dim};
    const RowSet vs{(uintptr_t)v, v_token_stride, v_head_stride, total_tokens, hkv, head_dim};
    if (!ks.apart() || !vs.apart() || ks.meets(vs))
        return fail(TA_ERR_INVALID_ARG, "%s: rows of k or v overlap", fn);
    const int64_t held = (num_pages * hkv) << lp, cache = held * head_dim * (q8 ? 1 : 2);
    for (const RowSet &x : {ks, vs}) {
        const Span spans[] = {{(const void *)x.at, 2 * x.extent()},
                              {k_cache, cache},
                              {v_cache, cache},
                              {k_scale, held},
                              {v_scale, held},
                              {block_table, 4LL * batch * table_width},
                              {cu, 4LL * batch + 4},
                              {starts, 4LL * batch}};
        if (spans_overlap(spans, 1, 8))
            return fail(TA_ERR_INVALID_ARG, "%s: an output overlaps another argument", fn);
    }
    ReadArgs a{};
    a.kc = k_cache;
    a.vc = v_cache;
    a.ks = static_cast<const uint8_t *>(k_scale);
    a.vs = static_cast<const uint8_t *>(v_scale);
    a.table = block_table;
    a.cu = cu;
    a.starts = starts;
    a.k = static_cast<uint16_t *>(k);
    a.v = static_cast<uint16_t *>(v);
    a.k_token = k_token_stride;
    a.k_head = k_head_stride;
    a.v_token = v_token_stride;
    a.v_head = v_head_stride;
    a.total_tokens = total_tokens;
    a.batch = batch;
    a.width = table_width;
    a.hkv = hkv;
    a.page_log2 = lp;
    a.num_pages = (int32_t)num_pages;
    a.blocks = (int32_t)((total_tokens + kReadTokens - 1) / kReadTokens);
    const int wgs = std::min(a.blocks, 1 << 22);  // a launch holds 2^32 threads
    const auto kernel = q8 ? (head_dim == 128 ? cache_read_kernel<128, true>
                                              : cache_read_kernel<64, true>)
                           : (head_dim == 128 ? cache_read_kernel<128, false>
                                              : cache_read_kernel<64, false>);
    hipLaunchKernelGGL(kernel, dim3((uint32_t)wgs), dim3(256), 0, static_cast<hipStream_t>(stream),
                       a);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess)
        return fail(TA_ERR_HIP, "%s: %s", fn, hipGetErrorString(err));
    return TA_OK;
}

extern "C" ta_status kv_cache_read(const void *k_cache, const void *v_cache,
                                   const int32_t *block_table, int32_t batch, int32_t table_width,
                                   const int32_t *cu, const int32_t *starts, void *k, void *v,
                                   int64_t k_token_stride, int64_t k_head_stride,
                                   int64_t v_token_stride, int64_t v_head_stride,
                                   int64_t total_tokens, int64_t num_pages, int32_t hkv,
                                   int32_t page_size, int32_t head_dim, void *stream)
{
    return cache_read("kv_cache_read", false, k_cache, nullptr, v_cache, nullptr, block_table,
                      batch, table_width, cu, starts, k, v, k_token_stride, k_head_stride,
                      v_token_stride, v_head_stride, total_tokens, num_pages, hkv, page_size,
                      head_dim, stream);
}

extern "C" ta_status kv_cache_read_q8(const void *k_cache, const void *k_scale,
                                      const void *v_cache, const void *v_scale,
                                      const int32_t *block_table, int32_t batch,
                                      int32_t table_width, const int32_t *cu,
                                      const int32_t *starts, void *k, void *v,
                                      int64_t k_token_stride, int64_t k_head_stride,
                                      int64_t v_token_stride, int64_t v_head_stride,
                                      int64_t total_tokens, int64_t num_pages, int32_t hkv,
                                      int32_t page_size, int32_t head_dim, void *stream)
{
    return cache_read("kv_cache_read_q8", true, k_cache, k_scale, v_cache, v_scale, block_table,
                      batch, table_width, cu, starts, k, v, k_token_stride, k_head_stride,
                      v_token_stride, v_head_stride, total_tokens, num_pages, hkv, page_size,
                      head_dim, stream);
}
