// Block tables and slot maps of a decoder step, built on the GPU from the requests' lengths (amap_cache_assign).
//
// Two prefix sums over the requests say everything: of fresh tokens (where a request's tokens begin) and of new pages (where
// its pages begin in the free list).  From them every token and every new page is found by itself: token t belongs to the
// last request that begins at or before t, and its page is an old entry of the table or, past those, an entry of
// the free list, so nothing is read that another workgroup writes and one launch does it all.  Each workgroup makes the sums for itself
// in LDS (8 bytes a request; reading them again costs less than a second launch), then takes its share of the tokens and pages.
// Bound by its launch: 64 requests of one token 3.1 us in the kernel (an empty one 2.5), 365 000 tokens of 389 prompts 6.3 us, of which their 5.9 MB are 1.
#include "amap_cache.hpp"

using namespace amap_cache_detail;
using namespace amap_detail;
using namespace amap_dev;

namespace {

constexpr int kAssignThreads = 512, kAssignWaves = kAssignThreads / 64;
constexpr int64_t kMaxRequests = 16384;   // two sums each in 128 KB of LDS

struct AssignArgs {
    const int32_t *cached, *fresh, *free_pages;
    int32_t *table, *begin, *length, *position, *owner, *taken;
    int64_t *slot;
    int64_t table_stride, n_tokens, n_free;
    uint32_t requests, page;
    int32_t width;
};

// how many pages of a row are there before the step, and after it
__device__ __forceinline__ void pages_of(const AssignArgs &a, uint32_t r, uint32_t &cached, uint32_t &fresh, uint32_t &have, uint32_t &need) {
    cached = a.cached ? (uint32_t)max(a.cached[r], 0) : 0u;
    fresh = (uint32_t)max(a.fresh[r], 0);
    const uint32_t w = (uint32_t)a.width;
    auto whole = [&](uint32_t tokens) { const uint32_t q = tokens / a.page; return q + (tokens != q * a.page); };
    have = min(whole(cached), w);
    need = max(have, min(whole(cached + fresh), w));
}

// inclusive sums over the workgroup of two values; `part` holds a pair per wavefront
__device__ __forceinline__ void block_sums(uint32_t &x, uint32_t &y, uint32_t (*part)[2]) {
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
#pragma unroll
    for (uint32_t d = 1; d < 64; d <<= 1) {
        const uint32_t u = __shfl_up(x, d), v = __shfl_up(y, d);
        if (lane >= d) x += u, y += v;
    }
    if (lane == 63) part[wave][0] = x, part[wave][1] = y;
    __syncthreads();
    for (uint32_t w = 0; w < wave; ++w) x += part[w][0], y += part[w][1];
}

// the last i in [0, n) with sums[i] <= at (sums[0] = 0)
__device__ __forceinline__ uint32_t last_at_or_before(const uint32_t *sums, uint32_t n, uint32_t at) {
    uint32_t lo = 0, hi = n;
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) >> 1;
        if (sums[mid] <= at)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}

__global__ __launch_bounds__(kAssignThreads) void amap_assign_kernel(const AssignArgs a) {
    extern __shared__ uint32_t sums[];
    __shared__ uint32_t part[kAssignWaves][2];
    const uint32_t n = a.requests, tid = threadIdx.x;
    uint32_t *const begin = sums, *const pages = sums + n + 1;
    uint32_t tokens_before = 0, pages_before = 0;
    for (uint32_t base = 0; base < n; base += kAssignThreads) {
        const uint32_t r = base + tid;
        uint32_t cached = 0, fresh = 0, have = 0, need = 0;
        if (r < n) pages_of(a, r, cached, fresh, have, need);
        uint32_t x = fresh, y = need - have;
        block_sums(x, y, part);
        if (r < n) {
            begin[r + 1] = tokens_before + x;
            pages[r + 1] = pages_before + y;
            if (blockIdx.x == 0) {
                a.begin[r + 1] = (int32_t)(tokens_before + x);
                a.length[r] = (int32_t)(cached + fresh);
            }
        }
        __syncthreads();
        const uint32_t last = min(base + kAssignThreads, n);
        if (tid == 0 && base == 0) begin[0] = pages[0] = 0;
        tokens_before = begin[last];
        pages_before = pages[last];
    }
    __syncthreads();
    if (blockIdx.x == 0 && tid == 0) {
        a.begin[0] = 0;
        a.taken[0] = (int32_t)pages_before;
    }
    const int64_t step = (int64_t)gridDim.x * kAssignThreads, first = (int64_t)blockIdx.x * kAssignThreads + tid;
    for (int64_t i = first; i < (int64_t)pages_before; i += step) {
        const uint32_t r = last_at_or_before(pages, n, (uint32_t)i);
        uint32_t cached, fresh, have, need;
        pages_of(a, r, cached, fresh, have, need);
        const uint32_t j = have + ((uint32_t)i - pages[r]);
        if (j < need) a.table[(int64_t)r * a.table_stride + j] = i < a.n_free ? a.free_pages[i] : -1;
    }
    for (int64_t t = first; t < a.n_tokens; t += step) {
        int64_t slot = -1;
        int32_t position = -1, owner = -1;
        if (t < (int64_t)tokens_before) {
            const uint32_t r = last_at_or_before(begin, n, (uint32_t)t);
            uint32_t cached, fresh, have, need;
            pages_of(a, r, cached, fresh, have, need);
            const uint32_t at = cached + ((uint32_t)t - begin[r]);
            owner = (int32_t)r;
            position = (int32_t)at;
            const uint32_t j = at / a.page;
            int32_t page = -1;
            if (j < have)
                page = a.table[(int64_t)r * a.table_stride + j];
            else if (j < need) {
                const int64_t i = (int64_t)pages[r] + (j - have);
                if (i < a.n_free) page = a.free_pages[i];
            }
            if (page >= 0) slot = (int64_t)page * a.page + (at - j * a.page);
        }
        a.slot[t] = slot;
        a.position[t] = position;
        a.owner[t] = owner;
    }
}

// Whether an array that the call writes meets another one of its arrays (outputs would be read as lengths by workgroups that come later).
bool any_meet(const amap_assign &a) {
    const int64_t rows = a.requests && a.table_width ? (a.requests - 1) * a.table_stride + a.table_width : 0;
    const Box all[] = {box_of(a.table, 4 * rows), box_of(a.begin, 4 * (a.requests + 1)), box_of(a.length, 4 * a.requests), box_of(a.slot, 8 * a.n_tokens), box_of(a.position, 4 * a.n_tokens),
                       box_of(a.owner, 4 * a.n_tokens), box_of(a.taken, 4), box_of(a.cached, a.cached ? 4 * a.requests : 0), box_of(a.fresh, 4 * a.requests), box_of(a.free_pages, 4 * a.n_free)};
    for (int i = 0; i < 7; ++i)
        for (int j = i + 1; j < 10; ++j)
            if (meet(all[i], all[j])) return true;
    return false;
}

}  // namespace

extern "C" amap_status amap_cache_assign(const amap_assign *a, void *stream) {
    if (!a || a->requests < 0 || a->n_tokens < 0 || a->n_free < 0 || a->page_size < 1 || a->table_width < 0) return AMAP_E_INVALID;
    if (!a->begin || !a->taken) return AMAP_E_INVALID;
    if (a->requests && (!a->fresh || !a->length || (a->table_width && !a->table))) return AMAP_E_INVALID;
    if (a->n_tokens && (!a->slot || !a->position || !a->owner)) return AMAP_E_INVALID;
    if (a->n_free && !a->free_pages) return AMAP_E_INVALID;
    if (a->requests > kMaxRequests) return refuse("more than 16384 requests in a step");
    if (a->n_tokens > INT32_MAX || (a->requests > 1 && a->table_stride < a->table_width)) return AMAP_E_SHAPE;
    if (a->requests && a->table_stride > ((int64_t)1 << 40)) return AMAP_E_SHAPE;
    if (a->n_free > ((int64_t)1 << 40)) return AMAP_E_SHAPE;
    if (any_meet(*a)) return AMAP_E_ALIAS;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const StreamDevice device(s);
    if (device.status() != hipSuccess) return launched(device.status(), "the stream's device");
    const uint32_t lds = 8u * ((uint32_t)a->requests + 1u);
    if (lds > 65536) {   // what a launch may ask for without it
        static LdsReservation reserved;
        const hipError_t e = reserved.on_current_device({reinterpret_cast<const void *>(amap_assign_kernel)}, 8 * ((int)kMaxRequests + 1));
        if (e != hipSuccess) return launched(e, "amap_assign_kernel: cannot reserve its LDS");
    }
    const AssignArgs g{a->cached, a->fresh, a->free_pages, a->table, a->begin, a->length, a->position, a->owner, a->taken, a->slot, a->table_stride, a->n_tokens,
                       a->n_free, (uint32_t)a->requests, (uint32_t)a->page_size, a->table_width};
    const int64_t most = 1024, wanted = (a->n_tokens + kAssignThreads - 1) / kAssignThreads;   // (what the chip holds at once)
    const uint32_t grid = (uint32_t)(wanted < 1 ? 1 : wanted > most ? most : wanted);
    return launched(launch_kernel<amap_assign_kernel>(dim3(grid), dim3(kAssignThreads), lds, s, g), "amap_assign_kernel");
}
