// C ABI of the paged cache: argument checks, layout, dispatch.  No device memory is allocated or freed here, and no device state is
// mirrored: what a call depends on is read by its kernels.
#include <math.h>
#include <stdlib.h>
#include <string.h>

#include <new>

#include "pod_paged.h"

static size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

namespace {
struct paged_layout {
    pod_layout ly;
    pod_paged_regions r;
    size_t off_flag, off_room, off_tickets, off_scratch, total;
};

// scratch of fork and compact: see pod_paged_kernels.hip
size_t scratch_ints(const pod_paged_config *cfg)
{
    const size_t fork = 8 + 4 * (size_t)kPagedMaxBatch, compact = 8 + 2 * ((size_t)cfg->num_pages + cfg->num_window_pages);
    return fork > compact ? fork : compact;
}

int make_paged_layout(const pod_paged_config *cfg, paged_layout *pl)
{
    if (!cfg) return pod_fail(POD_ERR_INVALID_ARG, "config is NULL");
    memset(pl, 0, sizeof *pl);
    if (const int rc = pod_make_layout(&cfg->base, &pl->ly)) return rc;
    const pod_layout &ly = pl->ly;
    if (ly.B > kPagedMaxBatch) return pod_fail(POD_ERR_INVALID_ARG, "a paged cache has at most %d slots, got max_batch %d", kPagedMaxBatch, ly.B);
    const int ps = cfg->page_size;
    if (ps < 16 || ps > 256 || (ps & (ps - 1))) return pod_fail(POD_ERR_INVALID_ARG, "page_size must be 16, 32, 64, 128 or 256, got %d", ps);
    if (ly.maxctx > (1 << 28)) return pod_fail(POD_ERR_INVALID_ARG, "max_context %d: at most 2^28 tokens", ly.maxctx);
    if (cfg->dtype != POD_TYPE_BF16 && cfg->dtype != POD_TYPE_FP16) return pod_fail(POD_ERR_INVALID_ARG, "unknown dtype %d", cfg->dtype);
    if (cfg->num_pages < 1 || cfg->num_pages > (1 << 26)) return pod_fail(POD_ERR_INVALID_ARG, "num_pages %d outside [1, 2^26]", cfg->num_pages);
    const int upper = ly.L * ly.Hkv - ly.nslots;
    if (cfg->num_window_pages > (1 << 26) || (upper ? cfg->num_window_pages < 1 : cfg->num_window_pages != 0))
        return pod_fail(POD_ERR_INVALID_ARG, "num_window_pages %d: %s", cfg->num_window_pages,
                        upper ? "upper layers keep keys in them, 1 to 2^26" : "no layer is an upper layer, must be 0");
    pod_paged_regions &r = pl->r;
    r.key_streams = ly.nslots; r.value_streams = ly.L * ly.Hkv; r.window_streams = upper;
    r.table_width = (ly.maxctx + ps - 1) / ps;
    const size_t np = cfg->num_pages, nw = cfg->num_window_pages, row = (size_t)ly.D * 2, table = (size_t)ly.B * r.table_width * 4;
    size_t off = 0;
    pl->off_flag = off; off += 256;
    pl->off_room = off; off = align_up(off + (size_t)ly.B * 4, 256);
    pl->off_tickets = off; off = align_up(off + (size_t)ly.B * ly.Hkv * 4, 256);
    pl->off_scratch = off; off = align_up(off + scratch_ints(cfg) * 4, 256);
    r.state = off;
    r.lens = off; off = align_up(off + (size_t)ly.B * 4, 256);
    r.page_refs = off; off = align_up(off + np * 4, 256);
    r.window_refs = off; off = align_up(off + nw * 4, 256);
    r.page_table = off; off = align_up(off + table, 256);
    r.window_table = off; off = align_up(off + table, 256);
    r.state_bytes = off - r.state;
    r.keys = off; off = align_up(off + (size_t)r.key_streams * np * ps * row, 256);
    r.values = off; off = align_up(off + (size_t)r.value_streams * np * ps * row, 256);
    r.window_keys = off; off = align_up(off + (size_t)r.window_streams * nw * ps * row, 256);
    pl->total = off;
    return POD_OK;
}

int check_rows(const void *p, int64_t stride, int heads, int d, const char *what)
{
    if (!p) return pod_fail(POD_ERR_INVALID_ARG, "%s is NULL", what);
    if ((uintptr_t)p % 16) return pod_fail(POD_ERR_INVALID_ARG, "%s must be 16-byte aligned", what);
    if (stride < (int64_t)heads * d || stride % 8 || stride > ((int64_t)1 << 40))
        return pod_fail(POD_ERR_INVALID_ARG, "%s: token stride %lld must be a multiple of 8 and at least %d x %d", what, (long long)stride, heads, d);
    return POD_OK;
}

int check_layer(const pod_paged *c, int layer)
{
    if (!c) return pod_fail(POD_ERR_INVALID_ARG, "cache is NULL");
    if (layer < 0 || layer >= c->v.L) return pod_fail(POD_ERR_INVALID_ARG, "layer %d outside [0, %d)", layer, c->v.L);
    return POD_OK;
}

int check_entries(const pod_paged *c, int n)
{
    if (!c) return pod_fail(POD_ERR_INVALID_ARG, "cache is NULL");
    if (n < 0 || n > c->v.B) return pod_fail(POD_ERR_INVALID_ARG, "%d entries, the cache has %d slots", n, c->v.B);
    return POD_OK;
}

int check_plan(const pod_paged *c, int n, int rows, const void *plan)
{
    if (const int rc = check_entries(c, n)) return rc;
    if (rows < 0 || rows > (1 << 28)) return pod_fail(POD_ERR_INVALID_ARG, "total_rows %d outside [0, 2^28]", rows);
    if (!plan || (uintptr_t)plan % 256) return pod_fail(POD_ERR_INVALID_ARG, "plan is NULL or not 256-byte aligned");
    return POD_OK;
}

// k and v of a call: both or none
int check_new(const pod_paged *c, const void *k, int64_t ks, const void *v, int64_t vs)
{
    if (!k != !v) return pod_fail(POD_ERR_INVALID_ARG, "k and v: both or none");
    if (!k) return POD_OK;
    if (const int rc = check_rows(k, ks, c->v.Hkv, c->v.D, "k")) return rc;
    return check_rows(v, vs, c->v.Hkv, c->v.D, "v");
}

int check_queries(const pod_paged *c, int layer, const void *q, int64_t qs, const void *q_shared, int64_t qss, float scale, const void *out)
{
    if (const int rc = check_rows(q, qs, c->v.Hq, c->v.D, "q")) return rc;
    if (!q_shared && !c->lowest_all[layer])
        return pod_fail(POD_ERR_INVALID_ARG, "layer %d is not the lowest of every head's block: q_shared must be given", layer);
    if (q_shared)
        if (const int rc = check_rows(q_shared, qss, c->v.Hq, c->v.D, "q_shared")) return rc;
    if (!(scale > 0.f) || !isfinite(scale)) return pod_fail(POD_ERR_INVALID_ARG, "scale must be positive and finite");
    if (!out || (uintptr_t)out % 16) return pod_fail(POD_ERR_INVALID_ARG, "out is NULL or not 16-byte aligned");
    return POD_OK;
}
} // namespace

pod_paged_plan_view pod_paged_plan_at(const void *plan, int rep, int n, int rows, size_t *bytes)
{
    pod_paged_plan_view p;
    const int64_t tokens = pod_paged_tile_tokens(rep);
    p.max_tiles = (int32_t)(rows / tokens + (n < rows ? n : rows));
    char *b = (char *)plan;
    size_t off = 0;
    p.head = (pod_paged_plan_head *)(b + off); off = align_up(off + sizeof(pod_paged_plan_head), 256);
    p.seq = (pod_paged_seq *)(b + off); off = align_up(off + (size_t)n * sizeof(pod_paged_seq), 256);
    p.row = (pod_paged_row *)(b + off); off = align_up(off + (size_t)rows * sizeof(pod_paged_row), 256);
    p.tile = (pod_paged_tile *)(b + off); off = align_up(off + (size_t)p.max_tiles * sizeof(pod_paged_tile), 256);
    if (bytes) *bytes = off;
    return p;
}

pod_paged_heads pod_paged_make_heads(const pod_paged *c, int layer)
{
    pod_paged_heads h;
    memset(&h, 0, sizeof h);
    for (int i = 0; i < c->v.Hkv; ++i) {
        h.key[i] = c->kstream[(size_t)layer * c->v.Hkv + i];
        h.window[i] = c->wstream[(size_t)layer * c->v.Hkv + i];
    }
    return h;
}

extern "C" int pod_paged_bytes(const pod_paged_config *cfg, size_t *bytes)
{
    if (!bytes) return pod_fail(POD_ERR_INVALID_ARG, "bytes is NULL");
    paged_layout pl;
    if (const int rc = make_paged_layout(cfg, &pl)) return rc;
    *bytes = pl.total;
    return POD_OK;
}

extern "C" int pod_paged_layout(const pod_paged_config *cfg, pod_paged_regions *regions)
{
    if (!regions) return pod_fail(POD_ERR_INVALID_ARG, "regions is NULL");
    paged_layout pl;
    if (const int rc = make_paged_layout(cfg, &pl)) return rc;
    *regions = pl.r;
    return POD_OK;
}

extern "C" int pod_paged_workspace_bytes(const pod_paged_config *cfg, size_t *bytes)
{
    if (!bytes) return pod_fail(POD_ERR_INVALID_ARG, "bytes is NULL");
    paged_layout pl;
    if (const int rc = make_paged_layout(cfg, &pl)) return rc;
    *bytes = pod_paged_decode_workspace(pl.ly);
    return POD_OK;
}

extern "C" int pod_paged_plan_bytes(const pod_paged_config *cfg, int n, int total_rows, size_t *bytes)
{
    if (!bytes) return pod_fail(POD_ERR_INVALID_ARG, "bytes is NULL");
    paged_layout pl;
    if (const int rc = make_paged_layout(cfg, &pl)) return rc;
    if (n < 0 || n > pl.ly.B) return pod_fail(POD_ERR_INVALID_ARG, "%d entries, the cache has %d slots", n, pl.ly.B);
    if (total_rows < 0 || total_rows > (1 << 28)) return pod_fail(POD_ERR_INVALID_ARG, "total_rows %d outside [0, 2^28]", total_rows);
    (void)pod_paged_plan_at(nullptr, pl.ly.rep, n, total_rows, bytes);
    return POD_OK;
}

extern "C" int pod_paged_destroy(pod_paged *cache)
{
    if (!cache) return POD_OK;
    free(cache->kstream);
    free(cache->wstream);
    free(cache->lowest_all);
    delete cache;
    return POD_OK;
}

extern "C" int pod_paged_init(const pod_paged_config *cfg, void *dev_buf, size_t bytes, void *stream, pod_paged **out)
{
    if (!out) return pod_fail(POD_ERR_INVALID_ARG, "out is NULL");
    *out = nullptr;
    paged_layout pl;
    if (const int rc = make_paged_layout(cfg, &pl)) return rc;
    if (!dev_buf) return pod_fail(POD_ERR_INVALID_ARG, "dev_buf is NULL");
    if ((uintptr_t)dev_buf % 256) return pod_fail(POD_ERR_INVALID_ARG, "dev_buf must be 256-byte aligned");
    if (bytes < pl.total) return pod_fail(POD_ERR_CAPACITY, "buffer has %zu bytes, cache needs %zu", bytes, pl.total);
    pod_paged *c = new (std::nothrow) pod_paged;
    if (!c) return pod_fail(POD_ERR_CAPACITY, "out of host memory");
    memset(c, 0, sizeof *c);
    const pod_layout &ly = pl.ly;
    const size_t LH = (size_t)ly.L * ly.Hkv;
    int32_t *lowest = nullptr;
    int nslots = 0;
    int rc = pod_make_tables(&cfg->base, &lowest, &c->kstream, &nslots, nullptr);
    if (rc) { delete c; return rc; }
    c->wstream = (int32_t *)malloc(LH * sizeof(int32_t));
    c->lowest_all = (bool *)malloc(ly.L * sizeof(bool));
    if (!c->wstream || !c->lowest_all) { free(lowest); pod_paged_destroy(c); return pod_fail(POD_ERR_CAPACITY, "out of host memory"); }
    int w = 0;
    for (int l = 0; l < ly.L; ++l) {
        c->lowest_all[l] = true;
        for (int h = 0; h < ly.Hkv; ++h) {
            const bool low = lowest[(size_t)l * ly.Hkv + h] == l;
            c->wstream[(size_t)l * ly.Hkv + h] = low ? -1 : w++;
            c->lowest_all[l] = c->lowest_all[l] && low;
        }
    }
    free(lowest);
    c->total_bytes = pl.total;
    c->dtype = cfg->dtype;
    pod_paged_view &v = c->v;
    v.base = (char *)dev_buf;
    v.flag = (int32_t *)(v.base + pl.off_flag);
    v.room = (int32_t *)(v.base + pl.off_room);
    v.tickets = (int32_t *)(v.base + pl.off_tickets);
    v.scratch = (int32_t *)(v.base + pl.off_scratch);
    v.lens = (int32_t *)(v.base + pl.r.lens);
    v.refs = (int32_t *)(v.base + pl.r.page_refs);
    v.wrefs = (int32_t *)(v.base + pl.r.window_refs);
    v.table = (int32_t *)(v.base + pl.r.page_table);
    v.wtable = (int32_t *)(v.base + pl.r.window_table);
    v.B = ly.B; v.ps = cfg->page_size; v.width = pl.r.table_width; v.np = cfg->num_pages; v.nw = cfg->num_window_pages; v.maxctx = ly.maxctx;
    v.S = ly.S; v.W = ly.W; v.L = ly.L; v.Hq = ly.Hq; v.Hkv = ly.Hkv; v.rep = ly.rep; v.D = ly.D;
    v.kstreams = pl.r.key_streams; v.vstreams = pl.r.value_streams; v.wstreams = pl.r.window_streams;
    v.off_keys = pl.r.keys; v.off_values = pl.r.values; v.off_wkeys = pl.r.window_keys;
    hipError_t e = hipGetDevice(&c->device);
    if (e == hipSuccess) e = hipDeviceGetAttribute(&c->cus, hipDeviceAttributeMultiprocessorCount, c->device);
    if (e != hipSuccess) { pod_paged_destroy(c); return pod_hip_fail(e, "hipGetDevice"); }
    rc = pod_launch_paged_reset(c, (hipStream_t)stream);
    if (rc) { pod_paged_destroy(c); return rc; }
    *out = c;
    return POD_OK;
}

extern "C" int pod_paged_reset(pod_paged *cache, void *stream)
{
    if (!cache) return pod_fail(POD_ERR_INVALID_ARG, "cache is NULL");
    return pod_launch_paged_reset(cache, (hipStream_t)stream);
}

extern "C" int pod_paged_check(pod_paged *cache, void *stream)
{
    if (!cache) return pod_fail(POD_ERR_INVALID_ARG, "cache is NULL");
    const hipStream_t st = (hipStream_t)stream;
    int32_t flag = 0;
    POD_HIP_TRY(hipMemcpyAsync(&flag, cache->v.flag, sizeof flag, hipMemcpyDeviceToHost, st));
    POD_HIP_TRY(hipStreamSynchronize(st));
    if (!flag) return POD_OK;
    if (const int rc = pod_launch_paged_clear(cache, st)) return rc;
    POD_HIP_TRY(hipStreamSynchronize(st));
    return pod_fail(POD_ERR_STATE, "a call was refused on the device:%s%s%s", flag & kPagedBadEntry ? " an entry that does not fit the cache's state;" : "",
                    flag & kPagedNoPages ? " too few free pages;" : "", flag & kPagedBadPlan ? " rows that do not fit the slots' tokens;" : "");
}

extern "C" int pod_paged_extend(pod_paged *cache, const int32_t *counts, const int32_t *slots, int n, void *stream)
{
    if (const int rc = check_entries(cache, n)) return rc;
    if (n == 0) return POD_OK;
    if (!counts) return pod_fail(POD_ERR_INVALID_ARG, "counts is NULL");
    return pod_launch_paged_extend(cache, counts, slots, n, (hipStream_t)stream);
}

extern "C" int pod_paged_fork(pod_paged *cache, const int32_t *src, const int32_t *dst, int n, void *stream)
{
    if (const int rc = check_entries(cache, n)) return rc;
    if (n == 0) return POD_OK;
    if (!src || !dst) return pod_fail(POD_ERR_INVALID_ARG, "src or dst is NULL");
    return pod_launch_paged_fork(cache, src, dst, n, (hipStream_t)stream);
}

extern "C" int pod_paged_free(pod_paged *cache, const int32_t *slots, int n, void *stream)
{
    if (const int rc = check_entries(cache, n)) return rc;
    if (n == 0) return POD_OK;
    if (!slots) return pod_fail(POD_ERR_INVALID_ARG, "slots is NULL");
    return pod_launch_paged_free(cache, slots, n, (hipStream_t)stream);
}

extern "C" int pod_paged_compact(pod_paged *cache, void *stream)
{
    if (!cache) return pod_fail(POD_ERR_INVALID_ARG, "cache is NULL");
    return pod_launch_paged_compact(cache, (hipStream_t)stream);
}

extern "C" int pod_paged_plan(pod_paged *cache, const int32_t *cu_rows, const int32_t *slots, int n, int total_rows, void *plan, size_t plan_bytes,
                              void *stream)
{
    if (const int rc = check_plan(cache, n, total_rows, plan)) return rc;
    if (!cu_rows) return pod_fail(POD_ERR_INVALID_ARG, "cu_rows is NULL");
    size_t need = 0;
    (void)pod_paged_plan_at(plan, cache->v.rep, n, total_rows, &need);
    if (plan_bytes < need) return pod_fail(POD_ERR_CAPACITY, "plan has %zu bytes, needs %zu", plan_bytes, need);
    return pod_launch_paged_plan(cache, cu_rows, slots, n, total_rows, plan, (hipStream_t)stream);
}

extern "C" int pod_paged_store(pod_paged *cache, int layer, const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                               int n, int total_rows, const void *plan, void *stream)
{
    if (const int rc = check_layer(cache, layer)) return rc;
    if (const int rc = check_plan(cache, n, total_rows, plan)) return rc;
    if (n == 0 || total_rows == 0) return POD_OK;
    if (!k) return pod_fail(POD_ERR_INVALID_ARG, "k is NULL");
    if (const int rc = check_new(cache, k, k_stride, v, v_stride)) return rc;
    return pod_launch_paged_store(cache, layer, k, k_stride, v, v_stride, n, total_rows, plan, (hipStream_t)stream);
}

extern "C" int pod_paged_prefill(pod_paged *cache, int layer, const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                                 const void *q, int64_t q_stride, const void *q_shared, int64_t q_shared_stride, int n, int total_rows,
                                 const void *plan, float scale, void *out, void *stream)
{
    if (const int rc = check_layer(cache, layer)) return rc;
    if (const int rc = check_plan(cache, n, total_rows, plan)) return rc;
    if (n == 0 || total_rows == 0) return POD_OK;
    if (const int rc = check_new(cache, k, k_stride, v, v_stride)) return rc;
    if (const int rc = check_queries(cache, layer, q, q_stride, q_shared, q_shared_stride, scale, out)) return rc;
    const hipStream_t st = (hipStream_t)stream;
    if (k)
        if (const int rc = pod_launch_paged_store(cache, layer, k, k_stride, v, v_stride, n, total_rows, plan, st)) return rc;
    pod_paged_call a;
    memset(&a, 0, sizeof a);
    a.layer = layer; a.n = n; a.rows = total_rows; a.q = q; a.q_stride = q_stride; a.qs = q_shared; a.qs_stride = q_shared_stride;
    a.scale = scale; a.out = out; a.plan = plan;
    return pod_launch_paged_prefill(cache, a, st);
}

extern "C" int pod_paged_decode(pod_paged *cache, int layer, const void *k_new, int64_t k_stride, const void *v_new, int64_t v_stride,
                                const void *q, int64_t q_stride, const void *q_shared, int64_t q_shared_stride, const int32_t *slots, int n,
                                float scale, void *workspace, size_t workspace_bytes, void *out, void *stream)
{
    if (const int rc = check_layer(cache, layer)) return rc;
    if (const int rc = check_entries(cache, n)) return rc;
    if (n == 0) return POD_OK;
    if (const int rc = check_new(cache, k_new, k_stride, v_new, v_stride)) return rc;
    if (const int rc = check_queries(cache, layer, q, q_stride, q_shared, q_shared_stride, scale, out)) return rc;
    pod_layout ly;
    memset(&ly, 0, sizeof ly);
    ly.rep = cache->v.rep; ly.D = cache->v.D;
    const size_t need = pod_paged_decode_workspace(ly);
    if (!workspace || (uintptr_t)workspace % 256) return pod_fail(POD_ERR_INVALID_ARG, "workspace is NULL or not 256-byte aligned");
    if (workspace_bytes < need) return pod_fail(POD_ERR_CAPACITY, "workspace has %zu bytes, needs %zu", workspace_bytes, need);
    pod_paged_call a;
    memset(&a, 0, sizeof a);
    a.layer = layer; a.n = n; a.rows = n; a.k = k_new; a.k_stride = k_stride; a.v = v_new; a.v_stride = v_stride;
    a.q = q; a.q_stride = q_stride; a.qs = q_shared; a.qs_stride = q_shared_stride; a.slots = slots;
    a.scale = scale; a.workspace = workspace; a.out = out;
    return pod_launch_paged_decode(cache, a, (hipStream_t)stream);
}
