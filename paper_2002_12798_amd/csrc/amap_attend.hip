// Attention of one new token per request over a paged cache (amap_cache_attend): s_i = scale q . k_i over the visible tokens,
// out = sum softmax(s)_i v_i, lse = log sum exp s_i, with the running maximum and sum of a softmax in one pass over the cache.
#include "amap_cache.hpp"

using namespace amap_cache_detail;
using namespace amap_detail;
using namespace amap_dev;

namespace {

struct AttendArgs {
    const char *k, *v, *q;
    char *out;
    float *lse;
    const float *k_scale, *v_scale;
    const int32_t *table, *length;
    int64_t table_stride, page_stride, token_stride, head_stride, q_token, q_head, out_token, out_head;
    uint32_t n_pages, page, width, dim, heads, group;
    FastDiv by_page, by_group;
    int32_t window;
    float scale;
};

__device__ __forceinline__ float value_of(amap_type type, const char *at, int64_t i) {
    if (type == AMAP_E4M3) return __builtin_amdgcn_cvt_f32_fp8((uint32_t)(uint8_t)at[i], 0);
    if (type == AMAP_BF16) return __uint_as_float((uint32_t) reinterpret_cast<const uint16_t *>(at)[i] << 16);
    return (float)reinterpret_cast<const _Float16 *>(at)[i];
}

// One wavefront per request and head, 64 tokens at a time: a lane has one token's score, then every fourth, 64th or so element of out.
template <amap_type TQ, amap_type TC>
__global__ __launch_bounds__(64) void amap_attend_kernel(const AttendArgs a) {
    const uint32_t r = blockIdx.x / a.heads, h = blockIdx.x - r * a.heads, kv = fdiv(h, a.by_group), lane = threadIdx.x;
    const int64_t most = (int64_t)a.width * a.page;
    const int64_t len = min((int64_t)max(a.length[r], 0), most);
    const int64_t first = a.window > 0 ? max(len - a.window, (int64_t)0) : 0;
    const char *const q = a.q + ((int64_t)r * a.q_token + (int64_t)h * a.q_head) * 2;
    float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    const float ks = a.scale * (a.k_scale ? a.k_scale[kv] : 1.f);
    for (int64_t base = first; base < len; base += 64) {
        const int64_t i = base + lane;
        int64_t off = -1;
        if (i < len) {
            const uint32_t j = fdiv((uint32_t)i, a.by_page);
            const int32_t id = a.table[(int64_t)r * a.table_stride + j];
            if (id >= 0 && (uint32_t)id < a.n_pages) off = (int64_t)id * a.page_stride + (int64_t)((uint32_t)i - j * a.page) * a.token_stride + (int64_t)kv * a.head_stride;
        }
        float s = -INFINITY;
        if (off >= 0) {
            s = 0.f;
            for (uint32_t d = 0; d < a.dim; ++d) s += value_of(TQ, q, d) * value_of(TC, a.k, off + d);
            s *= ks;
        }
        float top = s;
        for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
        top = fmaxf(m, top);
        const float base_of = top == -INFINITY ? 0.f : top, keep = expf(m - base_of);
        const float p = off >= 0 ? expf(s - base_of) : 0.f;
        float sum = p;
        for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
        l = l * keep + sum;
        m = top;
        for (int c = 0; c < 4; ++c) o[c] *= keep;
        for (int t = 0; t < 64; ++t) {
            const int64_t at = __shfl(off, t);
            const float w = __shfl(p, t);
            if (at < 0) continue;
            for (int c = 0; c < 4; ++c)
                if (lane + 64 * c < a.dim) o[c] += w * value_of(TC, a.v, at + lane + 64 * c);
        }
    }
    const bool none = m == -INFINITY && l == l && l == 0.f;
    const float by = none ? 0.f : (a.v_scale ? a.v_scale[kv] : 1.f) / l;
    char *const out = a.out + ((int64_t)r * a.out_token + (int64_t)h * a.out_head) * 2;
    for (uint32_t c = 0; c < 4; ++c) {
        const uint32_t d = lane + 64 * c;
        if (d >= a.dim) break;
        const float x = none ? 0.f : o[c] * by;
        reinterpret_cast<uint16_t *>(out)[d] = TQ == AMAP_BF16 ? __builtin_bit_cast(uint16_t, (__bf16)x) : __builtin_bit_cast(uint16_t, (_Float16)x);
    }
    if (a.lse && lane == 0) a.lse[(int64_t)r * a.heads + h] = none ? -INFINITY : m + logf(l);
}

amap_status check_attend(const amap_cache *cache, int heads, int64_t requests, int table_width) {
    Box k, v;
    const amap_status st = check_cache(cache, k, v);
    if (st != AMAP_OK) return st;
    if (heads < 1 || requests < 0 || table_width < 0) return AMAP_E_INVALID;
    if (heads % cache->kv_heads || requests > INT32_MAX / heads) return AMAP_E_SHAPE;
    if ((int64_t)table_width * cache->page_size > INT32_MAX) return AMAP_E_SHAPE;   // (lengths are int32)
    const int es = bytes_of(cache->type);
    if (cache->head_dim > 256 || cache->head_dim * es % 16) return refuse("head_dim over 256, or rows of the cache that are no whole 16-byte pieces");
    uint64_t at = reinterpret_cast<uintptr_t>(cache->k) | reinterpret_cast<uintptr_t>(cache->v);
    if (cache->n_pages > 1) at |= (uint64_t)cache->page_stride * es;
    if (cache->page_size > 1) at |= (uint64_t)cache->token_stride * es;
    if (cache->kv_heads > 1) at |= (uint64_t)cache->head_stride * es;
    return at % 16 ? refuse("rows of the cache that are not 16-byte aligned") : AMAP_OK;
}

}  // namespace

extern "C" amap_status amap_cache_attend_workspace(const amap_cache *cache, int heads, int64_t requests, int table_width, int64_t *bytes) {
    if (!bytes) return AMAP_E_INVALID;
    const amap_status st = check_attend(cache, heads, requests, table_width);
    if (st == AMAP_OK) *bytes = 0;
    return st;
}

extern "C" amap_status amap_cache_attend(const amap_cache *cache, const amap_heads *q, int64_t requests, const int32_t *table, int64_t table_stride, int table_width,
                                         const int32_t *length, float scale, int window, const amap_heads *out, float *lse, void *workspace, int64_t workspace_bytes,
                                         void *stream) {
    if (!q || !out) return AMAP_E_INVALID;
    amap_status st = check_attend(cache, q->heads, requests, table_width);
    if (st != AMAP_OK) return st;
    if (window < 0 || workspace_bytes < 0 || !std::isfinite(scale)) return AMAP_E_INVALID;
    if (requests == 0) return AMAP_OK;
    if (!length || (table_width && !table) || !q->data || !out->data) return AMAP_E_INVALID;
    if ((q->type != AMAP_BF16 && q->type != AMAP_F16) || out->type != q->type || (cache->type != q->type && cache->type != AMAP_E4M3)) return AMAP_E_INVALID;
    if (out->heads != q->heads || (requests > 1 && table_stride < table_width) || table_stride > ((int64_t)1 << 40)) return AMAP_E_SHAPE;
    const int dim = cache->head_dim;
    const Box from = box_of(*q, requests, dim), to = box_of(*out, requests, dim), k = box_of(*cache, cache->k), v = box_of(*cache, cache->v);
    if (!from.fits || !to.fits || !to.apart) return AMAP_E_SHAPE;
    if (meet(to, from) || meet(to, k) || meet(to, v)) return AMAP_E_ALIAS;
    if ((reinterpret_cast<uintptr_t>(q->data) | reinterpret_cast<uintptr_t>(out->data)) % 2) return refuse("a tensor that does not begin at a whole element");
    (void)workspace;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const StreamDevice device(s);
    if (device.status() != hipSuccess) return launched(device.status(), "the stream's device");
    const uint32_t group = (uint32_t)(q->heads / cache->kv_heads);
    const AttendArgs a{static_cast<const char *>(cache->k), static_cast<const char *>(cache->v), static_cast<const char *>(q->data), static_cast<char *>(out->data), lse,
                       cache->k_scale, cache->v_scale, table, length, table_stride, cache->page_stride, cache->token_stride, cache->head_stride, q->token_stride,
                       q->head_stride, out->token_stride, out->head_stride, (uint32_t)cache->n_pages, (uint32_t)cache->page_size, (uint32_t)table_width, (uint32_t)dim,
                       (uint32_t)q->heads, group, make_fastdiv((uint32_t)cache->page_size), make_fastdiv(group), window, scale};
    const dim3 grid((uint32_t)(requests * q->heads)), block(64);
    const bool bf = q->type == AMAP_BF16, wide = cache->type != AMAP_E4M3;
    return launched(bf ? wide ? launch_kernel<amap_attend_kernel<AMAP_BF16, AMAP_BF16>>(grid, block, 0, s, a) : launch_kernel<amap_attend_kernel<AMAP_BF16, AMAP_E4M3>>(grid, block, 0, s, a)
                  : wide ? launch_kernel<amap_attend_kernel<AMAP_F16, AMAP_F16>>(grid, block, 0, s, a)
                         : launch_kernel<amap_attend_kernel<AMAP_F16, AMAP_E4M3>>(grid, block, 0, s, a),
                    "amap_attend_kernel");
}
