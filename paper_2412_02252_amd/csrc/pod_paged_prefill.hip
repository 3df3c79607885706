// Attention of a packed batch's rows over the paged cache: the launches of pod_prefill_kernel.h with keys and values in pages.
//
// What bounds them is the matrix instructions, 4 D flops per (row, query head, key).  The tiles of all sequences are one list, longest first
// (paged_plan_kernel), whose length the host bounds by the rows alone: workgroups past its end leave at once.  4 documents of 2000 .. 8192 tokens x
// 32/8 heads x 128: 736 to 764 us from card to card, up to 1.0 PFLOP/s; 20 .. 700 tokens on 4096 .. 16384 held ones, 8 sequences: 419 to 432 us, up to 0.91
// (these launches alone; the stores before them take 26 and 7).
#include <mutex>

#include "pod_prefill_kernel.h"

int pod_launch_paged_prefill(const pod_paged *c, const pod_paged_call &a, hipStream_t st)
{
    const pod_paged_view &v = c->v;
    paged_prefill_params p = {};
    p.Hq = v.Hq; p.Hkv = v.Hkv; p.rep = v.rep; p.S = v.S; p.W = v.W;
    p.q = (const pod_bf16 *)a.q; p.qs = (const pod_bf16 *)a.qs;
    p.out = (pod_bf16 *)a.out;
    p.scale_log2e = a.scale * 1.4426950408889634f;
    p.c = v;
    p.plan = pod_paged_plan_at(a.plan, v.rep, a.n, a.rows, nullptr);
    p.q_stride = a.q_stride; p.qs_stride = a.qs_stride;
    p.nseq = a.n; p.rows = a.rows; p.layer = a.layer;
    p.heads = pod_paged_make_heads(c, a.layer);
#define POD_VARIANT(D, KS, E) {(const void *)prefill_kernel<D, kPaged, KS, E>, lds_bytes(D, KS)}
    static const struct { const void *fn; int lds; } variants[2][2][2] = { // [head dim 64 / 128][key groups - 1][type]
        {{POD_VARIANT(64, 1, type_bf16), POD_VARIANT(64, 1, type_fp16)}, {POD_VARIANT(64, 2, type_bf16), POD_VARIANT(64, 2, type_fp16)}},
        {{POD_VARIANT(128, 1, type_bf16), POD_VARIANT(128, 1, type_fp16)}, {POD_VARIANT(128, 2, type_bf16), POD_VARIANT(128, 2, type_fp16)}}};
#undef POD_VARIANT
    {   // raising the dynamic-LDS limit is needed once per device; any host thread may get here first
        static std::mutex attr_mutex;
        static bool attr_done[64] = {};
        int dev = -1;
        POD_HIP_TRY(hipGetDevice(&dev));
        if (dev < 0 || dev >= 64) return pod_fail(POD_ERR_INVALID_ARG, "device %d outside [0, 64)", dev);
        std::lock_guard<std::mutex> lock(attr_mutex);
        if (!attr_done[dev]) {
            for (const auto &by_dim : variants)
                for (const auto &by_groups : by_dim)
                    for (const auto &var : by_groups) POD_HIP_TRY(hipFuncSetAttribute(var.fn, hipFuncAttributeMaxDynamicSharedMemorySize, var.lds));
            attr_done[dev] = true;
        }
    }
    const int64_t wgs = (int64_t)p.plan.max_tiles * v.Hkv;
    if (wgs > 0x7fffffff) return pod_fail(POD_ERR_CAPACITY, "%d rows in one call are too many", a.rows);
    // Two key groups per tile where every workgroup has a CU of its own: the chain of key tiles is half as long, and there is nobody beside it to fill
    // its waits.  Only the rows are known here, not how much a sequence holds, so few rows on nothing pay for it.  One group / two, us with the stores,
    // upper layer, 32/8 x 128: 200 tokens on 8000 held (56 workgroups) 155 / 122, 1000 tokens (256) 35.8 / 34.3, 500 (128) 24.6 / 24.8, 110 (32) 13.4 / 14.9;
    // beyond: 1500 tokens (376) 49.8 / 50.2, 2000 (504) 61.3 / 64.5, 4 x 400 (432) 27.6 / 33.3.  16/4 x 64: 2 x 900 (232) 25.8 / 23.6, 4 x 1000 (516) 31.6 / 36.5.
    const int ks = wgs <= c->cus ? 2 : 1;
    const auto &var = variants[v.D == 128][ks - 1][c->dtype == POD_TYPE_FP16];
    void *args[] = {&p};
    POD_HIP_TRY(hipLaunchKernel(var.fn, dim3((unsigned)wgs), dim3(256 * ks), args, var.lds, st));
    POD_HIP_TRY(hipGetLastError());
    return POD_OK;
}
