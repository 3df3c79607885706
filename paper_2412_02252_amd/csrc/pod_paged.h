// Internal declarations of the paged cache (pod_paged*.hip).
#pragma once

#include "pod_internal.h"

constexpr int kPagedMaxBatch = 1024;     // slots: one thread of a bookkeeping workgroup each
constexpr int kPagedTileRows = 128;      // (token, query head of the group) rows of a prefill workgroup

// What kernels need of a cache, by value.  Device state is int32, see pod.h.
struct pod_paged_view {
    char *base;
    int32_t *flag, *lens, *refs, *wrefs, *table, *wtable;
    int32_t *room;                       // [max_batch] how many of a slot's last tokens may be written: kPagedAnyRoom, or what was made room for since an extend was refused
    int32_t *tickets;                    // [max_batch * Hkv] arrival counters of the decode launches, zero between launches
    int32_t *scratch;                    // fork and compact: see there
    int32_t B, ps, width, np, nw, maxctx, S, W, L, Hq, Hkv, rep, D;
    int32_t kstreams, vstreams, wstreams;
    size_t off_keys, off_values, off_wkeys;
};

// One layer's streams per kv head: where its distant logits' keys are, and its own keys (-1: the same, the layer is the block's lowest).
struct pod_paged_heads {
    int32_t key[kMaxKvHeads], window[kMaxKvHeads];
};

struct pod_paged {
    pod_paged_view v;
    int32_t dtype, device, cus;
    size_t total_bytes;
    int32_t *kstream, *wstream;          // [L][Hkv]
    bool *lowest_all;                    // [L]: no kv head of the layer has own keys in window pages
};

// A plan in device memory: header, sequences, rows, tiles.
struct pod_paged_plan_head { int32_t valid, ntiles, n, rows; };
struct pod_paged_seq { int32_t slot, len, first, row0; }; // tokens held, position of its first row, that row
struct pod_paged_row { int32_t slot, pos; };
struct pod_paged_tile { int32_t seq, token; };            // rows of sequence seq from its token-th on
struct pod_paged_plan_view {
    pod_paged_plan_head *head;
    pod_paged_seq *seq;
    pod_paged_row *row;
    pod_paged_tile *tile;
    int32_t max_tiles;                   // what the launch is sized for
};
// tokens of a tile
inline __host__ __device__ int pod_paged_tile_tokens(int rep) { return kPagedTileRows / rep; }
pod_paged_plan_view pod_paged_plan_at(const void *plan, int rep, int n, int rows, size_t *bytes);

int pod_launch_paged_reset(const pod_paged *c, hipStream_t st);
int pod_launch_paged_clear(const pod_paged *c, hipStream_t st); // the flag, and what refused extends left in room
int pod_launch_paged_extend(const pod_paged *c, const int32_t *counts, const int32_t *slots, int n, hipStream_t st);
int pod_launch_paged_fork(const pod_paged *c, const int32_t *src, const int32_t *dst, int n, hipStream_t st);
int pod_launch_paged_free(const pod_paged *c, const int32_t *slots, int n, hipStream_t st);
int pod_launch_paged_compact(const pod_paged *c, hipStream_t st);
int pod_launch_paged_plan(const pod_paged *c, const int32_t *cu, const int32_t *slots, int n, int rows, void *plan, hipStream_t st);
int pod_launch_paged_store(const pod_paged *c, int layer, const void *k, int64_t ks, const void *v, int64_t vs, int n, int rows,
                           const void *plan, hipStream_t st);
struct pod_paged_call { // of an attention call
    int layer, n, rows;
    const void *k, *v, *q, *qs;
    int64_t k_stride, v_stride, q_stride, qs_stride;
    const int32_t *slots;
    float scale;
    void *workspace, *out;
    const void *plan;
};
int pod_launch_paged_prefill(const pod_paged *c, const pod_paged_call &a, hipStream_t st);
int pod_launch_paged_decode(const pod_paged *c, const pod_paged_call &a, hipStream_t st);
size_t pod_paged_decode_workspace(const pod_layout &ly);
pod_paged_heads pod_paged_make_heads(const pod_paged *c, int layer);

constexpr int kPagedAnyRoom = 0x7fffffff;
constexpr int kPagedPlanValid = 0x706c616e; // head.valid of a plan that was made and not refused

enum { kPagedBadEntry = 1, kPagedNoPages = 2, kPagedBadPlan = 4 }; // bits of the sticky flag
