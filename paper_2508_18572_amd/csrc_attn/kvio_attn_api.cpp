// kvio_attn_api.cpp -- kvio_append and kvio_attend: their checks, and what they
// hand to the kernels.
#include <hip/hip_runtime.h>

#include <math.h>
#include <string.h>

#include <algorithm>

#include "kvio_attn.h"
#include "kvio_attn_internal.h"
#include "kvio_pool.h"

using kvio::fail;

namespace {

// A device array of `bytes` on the pool's GPU, `align`-aligned; null where `bytes` is 0.
kvio_status check_array(kvio_pool_t p, const void *ptr, uint64_t bytes, uintptr_t align, const char *fn, const char *what) {
    if (bytes == 0) return KVIO_OK;
    if (ptr == nullptr) return fail(KVIO_EINVAL, "%s: %s is null", fn, what);
    if ((reinterpret_cast<uintptr_t>(ptr) & (align - 1)) != 0)
        return fail(KVIO_EALIGN, "%s: %s is not %d-byte aligned", fn, what, int(align));
    const uint8_t *dev = nullptr;
    int device = -1;
    const kvio_status st = kvio::device_view(ptr, bytes, true, what, &dev, &device);
    if (st != KVIO_OK) return st;
    if (device != p->device) return fail(KVIO_EINVAL, "%s: %s lies on GPU %d, the pool on %d", fn, what, device, p->device);
    return KVIO_OK;
}

// Bytes from the first to one past the last of n rows of `row` bytes, `stride` elements of 2 bytes apart.
uint64_t reach(int64_t n, int64_t stride, int64_t row) { return n == 0 ? 0 : uint64_t(n - 1) * uint64_t(stride) * 2 + uint64_t(row); }

// An array of N rows of 16-bit elements, checked.
kvio_status check_rows(kvio_pool_t p, const void *ptr, int64_t n, int64_t stride, int64_t heads, int64_t dim, const char *fn, const char *what) {
    if (stride < heads * dim || stride % 8 != 0 || stride > (int64_t(1) << 40))
        return fail(KVIO_EINVAL, "%s: %s: tokens %lld elements apart; a multiple of 8, at least %lld is needed", fn, what, (long long)stride, (long long)(heads * dim));
    return check_array(p, ptr, reach(n, stride, heads * dim * 2), 16, fn, what);
}

// Whether two arrays of n rows of `row` bytes, `a_stride` and `b_stride` elements apart, may share memory.  Rows equally far
// apart (slices of one buffer) are looked at one by one, others as the whole ranges that they lie in.
bool overlaps(const void *a, int64_t a_stride, const void *b, int64_t b_stride, int64_t n, int64_t row) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    if (n == 0 || x >= y + reach(n, b_stride, row) || y >= x + reach(n, a_stride, row)) return false;
    if (n == 1 || a_stride != b_stride) return true;
    const uint64_t step = uint64_t(a_stride) * 2, off = (x > y ? x - y : y - x) % step;
    return off < uint64_t(row) || step - off < uint64_t(row);
}

kvio_status check_device(kvio_pool_t p, const char *fn) {
    int device = -1;
    const hipError_t e = hipGetDevice(&device);
    if (e != hipSuccess) return kvio::fail_hip(e, fn);
    if (device != p->device) return fail(KVIO_EINVAL, "%s: the pool lies on GPU %d, the current device is %d", fn, p->device, device);
    return KVIO_OK;
}

// Sizes, types and the pool: what needs no pointer.
kvio_status check_sizes(kvio_pool_t p, int32_t layer, const kvio_batch &b, int32_t dtype, int32_t cache_dtype, const char *fn) {
    if (p == nullptr) return fail(KVIO_EINVAL, "%s: null pool", fn);
    const kvio::PoolGeom &g = p->g;
    if (layer < 0 || layer >= g.num_layers) return fail(KVIO_EINVAL, "%s: layer %d outside [0, %d)", fn, layer, g.num_layers);
    if (dtype != KVIO_BF16 && dtype != KVIO_FP16) return fail(KVIO_EINVAL, "%s: dtype %d is neither KVIO_BF16 nor KVIO_FP16", fn, dtype);
    if (cache_dtype != dtype && cache_dtype != KVIO_E4M3)
        return fail(KVIO_EINVAL, "%s: cache_dtype %d is neither dtype nor KVIO_E4M3", fn, cache_dtype);
    const int elem = cache_dtype == KVIO_E4M3 ? 1 : 2;
    if (g.elem_bytes != elem)
        return fail(KVIO_EINVAL, "%s: cache_dtype %d takes %d bytes, the pool's elements have %d", fn, cache_dtype, elem, g.elem_bytes);
    if (b.num_seqs < 0 || b.num_tokens < 0 || b.max_query < 0)
        return fail(KVIO_EINVAL, "%s: negative num_seqs, num_tokens or max_query", fn);
    if (b.num_seqs == 0 || b.num_tokens == 0) return KVIO_OK;
    if (b.max_pages < 1 || b.table_stride < b.max_pages || b.table_stride > (int64_t(1) << 32))
        return fail(KVIO_EINVAL, "%s: max_pages %d must be >= 1 and table_stride %lld at least as many", fn, b.max_pages, (long long)b.table_stride);
    if (int64_t(b.max_pages) * g.page_size > INT32_MAX - 4096)
        return fail(KVIO_EINVAL, "%s: contexts of %d pages of %d tokens pass 2^31", fn, b.max_pages, g.page_size);
    if (b.q_start == nullptr && b.num_tokens < b.num_seqs)
        return fail(KVIO_EINVAL, "%s: without q_start %d sequences need as many tokens, not %d", fn, b.num_seqs, b.num_tokens);
    return KVIO_OK;
}

int32_t longest_query(const kvio_batch &b) {
    return b.q_start == nullptr ? 1 : b.max_query > 0 ? std::min(b.max_query, b.num_tokens) : b.num_tokens;
}

// The batch's and the cache's arrays; fills in what kernels see of them.
kvio_status check_cache(kvio_pool_t p, int32_t layer, const kvio_batch &b, bool e4m3, const float *k_scale, const float *v_scale,
                        int64_t scale_stride, const char *fn, kvio::CacheArgs *c) {
    const kvio::PoolGeom &g = p->g;
    kvio_status st = check_device(p, fn);
    const uint64_t table = (uint64_t(b.num_seqs - 1) * uint64_t(b.table_stride) + uint64_t(b.max_pages)) * 4;
    if (st == KVIO_OK) st = check_array(p, b.page_table, table, 4, fn, "page_table");
    if (st == KVIO_OK) st = check_array(p, b.ctx_len, uint64_t(b.num_seqs) * 4, 4, fn, "ctx_len");
    if (st == KVIO_OK && b.q_start != nullptr) st = check_array(p, b.q_start, (uint64_t(b.num_seqs) + 1) * 4, 4, fn, "q_start");
    const int64_t num_pages = g.num_slots / g.page_size;
    if (st == KVIO_OK && e4m3) {
        if (scale_stride < g.num_heads || scale_stride > (int64_t(1) << 32))
            return fail(KVIO_EINVAL, "%s: scale_stride %lld below the pool's %d heads", fn, (long long)scale_stride, g.num_heads);
        const uint64_t bytes = (uint64_t(num_pages - 1) * uint64_t(scale_stride) + uint64_t(g.num_heads)) * 4;
        st = check_array(p, k_scale, bytes, 4, fn, "k_scale");
        if (st == KVIO_OK) st = check_array(p, v_scale, bytes, 4, fn, "v_scale");
    }
    if (st != KVIO_OK) return st;
    memset(c, 0, sizeof *c);
    c->page_table = b.page_table;
    c->ctx_len = b.ctx_len;
    c->q_start = b.q_start;
    c->err = p->d_err;
    c->k_cache = p->layers[size_t(layer)];
    c->v_cache = p->layers[size_t(g.num_layers) + layer];
    c->k_scale = const_cast<float *>(k_scale);
    c->v_scale = const_cast<float *>(v_scale);
    c->scale_stride = scale_stride;
    c->table_stride = b.table_stride;
    c->num_seqs = b.num_seqs;
    c->num_tokens = b.num_tokens;
    c->max_query = longest_query(b);
    c->max_ctx = b.max_pages * g.page_size;
    c->num_pages = static_cast<int32_t>(num_pages);
    c->page_size = g.page_size;
    c->page_div = kvio::divider(g.page_size);
    c->heads = g.num_heads;
    c->head_dim = static_cast<int32_t>(g.seg_bytes / g.elem_bytes);
    return KVIO_OK;
}

constexpr float kLog2E = 1.44269504088896340736f;

// Rows of a KV head that kvio_attend_steps.hip holds in a wave's registers, by the size of heads.
int64_t most_step_rows(int64_t dim) { return dim <= 128 ? 64 : 32; }

kvio_status check_attend(kvio_pool_t p, int32_t layer, const kvio_attend_args *args, const char *fn) {
    if (args == nullptr) return fail(KVIO_EINVAL, "%s: null arguments", fn);
    const kvio_status st = check_sizes(p, layer, args->batch, args->dtype, args->cache_dtype, fn);
    if (st != KVIO_OK) return st;
    const int64_t dim = p->g.seg_bytes / p->g.elem_bytes;
    if (dim != 64 && dim != 128 && dim != 256) return fail(KVIO_EINVAL, "%s: heads of %lld dims; 64, 128 and 256 are built", fn, (long long)dim);
    if (args->num_q_heads < p->g.num_heads || args->num_q_heads % p->g.num_heads != 0 || args->num_q_heads > 65536)
        return fail(KVIO_EINVAL, "%s: %d query heads are no multiple of the pool's %d", fn, args->num_q_heads, p->g.num_heads);
    const int32_t group = args->num_q_heads / p->g.num_heads;
    if (group > kvio::block_rows(static_cast<int>(dim)))
        return fail(KVIO_EINVAL, "%s: %d query heads to a KV head; up to %d are built", fn, group, kvio::block_rows(static_cast<int>(dim)));
    if (args->window < 0) return fail(KVIO_EINVAL, "%s: window %d < 0", fn, args->window);
    if (!(args->softmax_scale > 0) || !isfinite(args->softmax_scale * kLog2E))
        return fail(KVIO_EINVAL, "%s: softmax_scale must be positive, and finite times log2(e)", fn);
    if (args->reserved != 0) return fail(KVIO_EINVAL, "%s: reserved is not 0", fn);
    const int64_t tiles = (int64_t(args->batch.max_pages) * p->g.page_size + 63) / 32;
    if (args->batch.num_seqs > 0 && args->batch.num_tokens > 0 && tiles * args->batch.num_seqs > INT32_MAX - 4096)
        return fail(KVIO_EINVAL, "%s: %d contexts of up to %d pages: too many tokens to count", fn, args->batch.num_seqs, args->batch.max_pages);
    // a wave for each when partial results are joined, and fewer than 2^32 threads to a launch
    const bool few = int64_t(longest_query(args->batch)) * group <= most_step_rows(dim);
    if (int64_t(args->batch.num_tokens) * args->num_q_heads > (few ? (1 << 26) - 4 : INT32_MAX))
        return fail(KVIO_EINVAL, "%s: %d tokens of %d heads: too many rows to count", fn, args->batch.num_tokens, args->num_q_heads);
    return KVIO_OK;
}

kvio::AttendPlan plan_of(kvio_pool_t p, const kvio_attend_args &args) {
    const kvio::PoolGeom &g = p->g;
    const int32_t dim = static_cast<int32_t>(g.seg_bytes / g.elem_bytes), longest = longest_query(args.batch), max_ctx = args.batch.max_pages * g.page_size;
    if (int64_t(longest) * (args.num_q_heads / g.num_heads) <= most_step_rows(dim))
        return kvio::plan_steps(args.cache_dtype == KVIO_E4M3, g.num_heads, args.num_q_heads, dim, args.batch, longest, max_ctx);
    return kvio::plan_blocks(g.num_heads, args.num_q_heads, dim, args.batch, longest, max_ctx);
}

}  // namespace

extern "C" {

kvio_status kvio_append(kvio_pool_t p, int32_t layer, const kvio_append_args *args, hipStream_t stream) {
    const char *fn = "kvio_append";
    kvio::clear_error();
    if (args == nullptr) return fail(KVIO_EINVAL, "%s: null arguments", fn);
    const kvio_batch &b = args->batch;
    kvio_status st = check_sizes(p, layer, b, args->dtype, args->cache_dtype, fn);
    if (st != KVIO_OK) return st;
    const int64_t H = p->g.num_heads, D = p->g.seg_bytes / p->g.elem_bytes, N = b.num_tokens;
    if (D % 16 != 0) return fail(KVIO_EINVAL, "%s: heads of %lld dims are no multiple of 16", fn, (long long)D);
    if (D > 1024) return fail(KVIO_EINVAL, "%s: heads of %lld dims; up to 1024 are built", fn, (long long)D);
    if (args->rot_dim < 0 || args->rot_dim > D || args->rot_dim % 16 != 0)
        return fail(KVIO_EINVAL, "%s: rot_dim %d must be a multiple of 16 up to %lld", fn, args->rot_dim, (long long)D);
    if ((args->flags & ~KVIO_APPEND_INTERLEAVED) != 0) return fail(KVIO_EINVAL, "%s: unknown flags 0x%x", fn, args->flags);
    if (args->reserved != 0) return fail(KVIO_EINVAL, "%s: reserved is not 0", fn);
    const bool with_q = args->q != nullptr;
    if (with_q ? args->num_q_heads < 1 || args->num_q_heads > 65536 : args->num_q_heads != 0 || args->q_out != nullptr)
        return fail(KVIO_EINVAL, "%s: num_q_heads %d and q_out do not fit q", fn, args->num_q_heads);
    if (b.num_seqs == 0 || N == 0) return KVIO_OK;
    const bool e4m3 = args->cache_dtype == KVIO_E4M3;
    kvio::AppendArgs a;
    st = check_cache(p, layer, b, e4m3, args->k_scale, args->v_scale, args->scale_stride, fn, &a.c);
    if (st == KVIO_OK) st = check_rows(p, args->k, N, args->k_stride, H, D, fn, "k");
    if (st == KVIO_OK) st = check_rows(p, args->v, N, args->v_stride, H, D, fn, "v");
    if (st == KVIO_OK && with_q) st = check_rows(p, args->q, N, args->q_stride, args->num_q_heads, D, fn, "q");
    if (st == KVIO_OK && with_q) st = check_rows(p, args->q_out, N, args->q_out_stride, args->num_q_heads, D, fn, "q_out");
    if (st == KVIO_OK && args->rot_dim > 0) st = check_array(p, args->inv_freq, uint64_t(args->rot_dim) * 2, 4, fn, "inv_freq");
    if (st == KVIO_OK && args->positions != nullptr) st = check_array(p, args->positions, uint64_t(N) * 4, 4, fn, "positions");
    if (st != KVIO_OK) return st;
    if (with_q && !(args->q_out == args->q && args->q_out_stride == args->q_stride) &&
        overlaps(args->q_out, args->q_out_stride, args->q, args->q_stride, N, args->num_q_heads * D * 2))
        return fail(KVIO_EINVAL, "%s: q_out overlaps q without being it", fn);
    a.k = static_cast<const uint8_t *>(args->k);
    a.v = static_cast<const uint8_t *>(args->v);
    a.q = static_cast<const uint8_t *>(args->q);
    a.q_out = static_cast<uint8_t *>(args->q_out);
    a.k_stride = args->k_stride * 2;
    a.v_stride = args->v_stride * 2;
    a.q_stride = args->q_stride * 2;
    a.q_out_stride = args->q_out_stride * 2;
    a.inv_freq = args->inv_freq;
    a.positions = args->positions;
    a.q_heads = args->num_q_heads;
    a.rot_half = args->rot_dim / 2;
    a.interleaved = (args->flags & KVIO_APPEND_INTERLEAVED) != 0;
    a.page_items = static_cast<int32_t>(std::min(N, N / p->g.page_size + 2 * int64_t(b.num_seqs)));
    if (kvio::append_threads(a, e4m3) >= int64_t(1) << 32) return fail(KVIO_EINVAL, "%s: %lld tokens are too many for one call", fn, (long long)N);
    const hipError_t e = kvio::launch_append(a, args->dtype, e4m3, stream);
    return e == hipSuccess ? KVIO_OK : kvio::fail_hip(e, fn);
}

kvio_status kvio_attend_workspace(kvio_pool_t p, const kvio_attend_args *args, size_t *bytes) {
    const char *fn = "kvio_attend_workspace";
    kvio::clear_error();
    if (bytes == nullptr) return fail(KVIO_EINVAL, "%s: null bytes", fn);
    const kvio_status st = check_attend(p, 0, args, fn);
    if (st != KVIO_OK) return st;
    *bytes = 0;
    if (args->batch.num_seqs == 0 || args->batch.num_tokens == 0) return KVIO_OK;
    *bytes = size_t(plan_of(p, *args).bytes);
    return KVIO_OK;
}

kvio_status kvio_attend(kvio_pool_t p, int32_t layer, const kvio_attend_args *args, hipStream_t stream) {
    const char *fn = "kvio_attend";
    kvio::clear_error();
    kvio_status st = check_attend(p, layer, args, fn);
    if (st != KVIO_OK) return st;
    const kvio_batch &b = args->batch;
    const int64_t D = p->g.seg_bytes / p->g.elem_bytes, N = b.num_tokens, Hq = args->num_q_heads;
    if (b.num_seqs == 0 || N == 0) return KVIO_OK;
    const bool e4m3 = args->cache_dtype == KVIO_E4M3;
    kvio::AttendArgs a;
    st = check_cache(p, layer, b, e4m3, args->k_scale, args->v_scale, args->scale_stride, fn, &a.c);
    if (st == KVIO_OK) st = check_rows(p, args->q, N, args->q_stride, Hq, D, fn, "q");
    if (st == KVIO_OK) st = check_rows(p, args->out, N, args->out_stride, Hq, D, fn, "out");
    if (st == KVIO_OK && args->lse != nullptr) st = check_array(p, args->lse, uint64_t(N) * uint64_t(Hq) * 4, 4, fn, "lse");
    if (st != KVIO_OK) return st;
    if (overlaps(args->out, args->out_stride, args->q, args->q_stride, N, Hq * D * 2))
        return fail(KVIO_EINVAL, "%s: out overlaps q", fn);
    a.q = static_cast<const uint8_t *>(args->q);
    a.out = static_cast<uint8_t *>(args->out);
    a.lse = args->lse;
    a.q_stride = args->q_stride * 2;
    a.out_stride = args->out_stride * 2;
    a.q_heads = args->num_q_heads;
    a.group = args->num_q_heads / p->g.num_heads;
    a.window = args->window < a.c.max_ctx ? args->window : 0;      // a longer one hides nothing
    a.scale_log2 = args->softmax_scale * kLog2E;
    a.group_div = kvio::divider(a.group);
    const kvio::AttendPlan plan = plan_of(p, *args);
    a.partials = static_cast<float *>(args->workspace);
    a.heads_per_group = plan.heads_per_group;
    a.workers = plan.workers;
    a.min_tiles = plan.min_tiles;
    a.slot_rows = plan.slot_rows;
    a.block_tokens = plan.block_tokens;
    a.min_keys = plan.min_keys;
    a.joined = plan.joined;
    a.join_rows = plan.join_rows;
    if (args->workspace_bytes < plan.bytes)
        return fail(KVIO_EINVAL, "%s: workspace of %llu bytes, %llu are needed", fn, (unsigned long long)args->workspace_bytes, (unsigned long long)plan.bytes);
    st = check_array(p, args->workspace, plan.bytes, 16, fn, "workspace");
    if (st != KVIO_OK) return st;
    const hipError_t e = (plan.few ? kvio::launch_steps : kvio::launch_blocks)(a, plan, args->dtype, e4m3, stream);
    return e == hipSuccess ? KVIO_OK : kvio::fail_hip(e, fn);
}

}  // extern "C"
