// Pages of the paged cache: taking, sharing, copying, packing and giving them back, and rows into pages.
//
// What a call decides (which pages) depends on all tables and counts at once and is a few thousand integers: one workgroup of 1024
// threads does it, an entry per thread, pages by the thousand, with prefix sums over the workgroup.  The result is the same however
// threads interleave: the lowest free page goes to the first (entry, token) that needs one.  What follows from it (rows and tables to
// copy) is spread over the chip by a second launch that reads the decision from the cache's scratch memory.
// Latency bounds the decisions (4 to 8 us each, a few dependent loads and prefix sums), the copy rate what follows: 64 forks of 8 prompts in 8 layers copy
// 140 MB, read and written, in 22 us; compaction of 16 documents' cache after 8 ended moves 708 MB in 137 to 139 us (5.1 TB/s).
#include "pod_paged.h"

namespace {

constexpr int kBook = 1024; // threads of a bookkeeping workgroup

__device__ inline int lane_id() { return threadIdx.x & 63; }

// Exclusive prefix sum over the workgroup and the total.  Called by all threads; what they wrote to memory and LDS before, all see after.
// With a cap < 2^30, and no x above it, sums stop at it: the total is right below it, and so are the prefix sums if it is.
__device__ __forceinline__ int block_scan(int x, int *total, int cap = 0x7fffffff)
{
    __shared__ int sums[kBook / 64];
    int incl = x;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int y = __shfl_up(incl, off);
        if (lane_id() >= off) incl = min(incl + y, cap);
    }
    __syncthreads(); // (the last call's sums have been read)
    if (lane_id() == 63) sums[threadIdx.x >> 6] = incl;
    __syncthreads();
    int before = 0, all = 0;
    for (int w = 0; w < (int)blockDim.x / 64; ++w) {
        const int s = sums[w];
        if (w < (int)threadIdx.x >> 6) before = min(before + s, cap);
        all = min(all + s, cap);
    }
    *total = all;
    return before + incl - x;
}

// Reference counts are read past the vector L1, which this launch's own atomics do not update.
__device__ inline int load_ref(const int32_t *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// A pool's pages as a workgroup walks them: every thread has up to 32 neighbouring ones and keeps what it asked of each in a bit, so that one
// read of the counts and one prefix sum answer for 32768 pages; larger pools are walked in pieces of that many.
constexpr int kPieceBits = 32;
struct page_piece {
    int first, per;                      // this thread's pages are first .. first + per - 1
    unsigned bits;
};
template <class F>
__device__ __forceinline__ page_piece read_piece(const int32_t *refs, int np, int base, F &&is_one)
{
    page_piece p;
    p.per = min((min(np - base, kPieceBits * kBook) + 4 * kBook - 1) / (4 * kBook) * 4, kPieceBits);
    p.first = base + (int)threadIdx.x * p.per;
    p.bits = 0;
    for (int k = 0; k < p.per; k += 4) {
        int r[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) r[x] = load_ref(refs + min(p.first + k + x, np - 1));
#pragma unroll
        for (int x = 0; x < 4; ++x) p.bits |= (unsigned)(p.first + k + x < np && is_one(p.first + k + x, r[x])) << (k + x);
    }
    return p;
}

// The free pages of a pool, the lowest first.
struct free_list {
    const int32_t *refs;
    int np, total, rank;                 // all of them; those of the first piece before this thread's
    page_piece piece;                    // the first one
    static __device__ __forceinline__ page_piece read(const int32_t *refs, int np, int base)
    {
        return read_piece(refs, np, base, [](int, int r) { return r == 0; });
    }
    // The constructor only asks for the first piece, count() needs it: whatever comes in between waits beside it.
    __device__ __forceinline__ free_list(const int32_t *refs_, int np_) : refs(refs_), np(np_), total(0), rank(0)
    {
        piece = np ? read(refs, np, 0) : page_piece{0, 0, 0};
    }
    __device__ __forceinline__ void count()
    {
        if (np == 0) return;
        rank = block_scan(__popc(piece.bits), &total);
        int more = 0, sum = 0;
        for (int base = kPieceBits * kBook; base < np; base += kPieceBits * kBook) more += __popc(read(refs, np, base).bits);
        if (np > kPieceBits * kBook) { block_scan(more, &sum); total += sum; }
    }
    template <class F>
    __device__ __forceinline__ void take(int want, F &&f) // f(rank, page) for the first `want`, by the thread that has the page
    {
        page_piece p = piece;
        int at = rank;
        for (int base = 0, done = 0;;) {
            for (unsigned b = p.bits; b && at < want; b &= b - 1, ++at) f(at, p.first + __ffs(b) - 1);
            base += kPieceBits * kBook;
            if (base >= np) return;
            int found;
            if (base == kPieceBits * kBook) block_scan(__popc(p.bits), &done); // the first piece's
            if (done >= want) return;
            p = read(refs, np, base);
            at = done + block_scan(__popc(p.bits), &found);
            done += found;
        }
    }
};

// Marks slots; true where the slot was marked before.
__device__ inline bool mark(unsigned *bits, int slot) { return atomicOr(bits + (slot >> 5), 1u << (slot & 31)) >> (slot & 31) & 1; }

__global__ void paged_reset_kernel(pod_paged_view c)
{
    const size_t at = (size_t)blockIdx.x * blockDim.x + threadIdx.x, step = (size_t)gridDim.x * blockDim.x;
    const size_t table = (size_t)c.B * c.width;
    for (size_t i = at; i < table; i += step) { c.table[i] = -1; c.wtable[i] = -1; }
    for (size_t i = at; i < (size_t)c.np; i += step) c.refs[i] = 0;
    for (size_t i = at; i < (size_t)c.nw; i += step) c.wrefs[i] = 0;
    for (size_t i = at; i < (size_t)c.B; i += step) { c.lens[i] = 0; c.room[i] = kPagedAnyRoom; }
    for (size_t i = at; i < (size_t)c.B * c.Hkv; i += step) c.tickets[i] = 0;
    if (at == 0) *c.flag = 0;
}

__global__ __launch_bounds__(kBook) void paged_clear_kernel(pod_paged_view c)
{
    if ((int)threadIdx.x < c.B) c.room[threadIdx.x] = kPagedAnyRoom;
    if (threadIdx.x == 0) *c.flag = 0;
}

// ---- extend.  A refused one leaves its entries without room (c.room): the length has not grown, so what follows in the same step would
// write its rows over tokens that are held, in pages that other slots may share.

__global__ __launch_bounds__(kBook) void paged_extend_kernel(pod_paged_view c, const int32_t *counts, const int32_t *slots, int n)
{
    __shared__ unsigned seen[kPagedMaxBatch / 32];
    __shared__ int before[kBook + 1], first[kBook], slot_of[kBook], held_of[kBook]; // held_of: tokens before, of entries that get more; else 0
    const int e = threadIdx.x;
    if (e < kPagedMaxBatch / 32) seen[e] = 0;
    __syncthreads();
    int slot = 0, len = 0, count = 0, bad = 0, room = 0;
    bool inside = false;
    if (e < n) {
        slot = slots ? slots[e] : e;
        count = counts[e];
        inside = slot >= 0 && slot < c.B;
        bad = !inside || count < 0;
        if (!bad) {
            len = c.lens[slot];
            room = c.room[slot];
            bad = mark(seen, slot) || len < 0 || len > c.maxctx || count > c.maxctx - len;
        }
    }
    if (__syncthreads_or(bad)) {
        if (inside && count != 0) c.room[slot] = 0;
        if (e == 0) atomicOr(c.flag, kPagedBadEntry);
        return;
    }
    slot_of[e] = slot;
    // (no more than one page above the pool: 1024 entries may want 2^24 pages each; where even so the sum could pass 32 bits it stops there too, for 0.3 us)
    const int have = (len + c.ps - 1) / c.ps, need = count > 0 ? min((len + count + c.ps - 1) / c.ps - have, c.np + 1) : 0;
    first[e] = have;
    held_of[e] = count > 0 ? len : 0;
    int total;
    before[e] = (int64_t)n * (c.np + 1) > 0x7fffffff ? block_scan(need, &total, c.np + 1) : block_scan(need, &total);
    if (e == 0) before[kBook] = total;
    __syncthreads();
    if (c.nw) {
        // Window pages with no token that position `len` still attends by its own layer's keys (j < S or j > len - W).  They are
        // given back oldest first, so the ones that are gone already lie below the rest: a wave per entry walks down to the first.
        const int lo = (c.S + c.ps - 1) / c.ps;
        for (int x = threadIdx.x >> 6; x < n; x += kBook / 64) {
            const int s = slot_of[x], held = held_of[x];
            const int end = held - c.W + 1 > 0 ? (held - c.W + 1) / c.ps : 0; // pages below hold positions <= held - W only
            for (int top = end; top > lo; top -= 64) {
                const int i = top - 1 - lane_id();
                int32_t *const entry = c.wtable + (size_t)s * c.width + i;
                const int page = i >= lo ? *entry : -1;
                if (page >= 0) {
                    *entry = -1;
                    if (page < c.nw) atomicSub(c.wrefs + page, 1);
                }
                if (__any(page < 0)) break;
            }
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); // this wave's counts are in memory before anybody reads them
        __syncthreads();
    }
    if (total > 0) {
        free_list pages(c.refs, c.np), wpages(c.wrefs, c.nw);
        pages.count();
        wpages.count();
        if (pages.total < total || (c.nw && wpages.total < total)) {
            if (inside && count > 0) c.room[slot] = 0;
            if (e == 0) atomicOr(c.flag, kPagedNoPages);
            return;
        }
        // rank r of the pages taken belongs to the entry x with before[x] <= r < before[x + 1]
        auto entry_of = [&](int32_t *table, int r) {
            int a = 0, b = kBook; // before[a] <= r < before[b]
            while (b - a > 1) {
                const int m = (a + b) / 2;
                if (before[m] <= r) a = m;
                else b = m;
            }
            return table + (size_t)slot_of[a] * c.width + first[a] + (r - before[a]);
        };
        pages.take(total, [&](int r, int page) { *entry_of(c.table, r) = page; c.refs[page] = 1; });
        if (c.nw) wpages.take(total, [&](int r, int page) { *entry_of(c.wtable, r) = page; c.wrefs[page] = 1; });
    }
    if (e < n) {
        c.lens[slot] = len + count;
        if (room != kPagedAnyRoom) c.room[slot] = room + count; // (never above the length)
    }
}

// ---- fork.  scratch: [0] entries (0: refused), from 8 on per entry: context page from, to, window page from, to (-1: none)

__global__ __launch_bounds__(kBook) void paged_fork_plan_kernel(pod_paged_view c, const int32_t *src, const int32_t *dst, int n)
{
    __shared__ unsigned is_src[kPagedMaxBatch / 32], is_dst[kPagedMaxBatch / 32];
    __shared__ int entry_of[kBook], dst_of[kBook], at_of[kBook]; // of the r-th partly filled page: the entry; of an entry: slot and place in its table
    const int e = threadIdx.x;
    free_list pages(c.refs, c.np), wpages(c.wrefs, c.nw);
    if (e < kPagedMaxBatch / 32) is_src[e] = is_dst[e] = 0;
    __syncthreads();
    int s = 0, d = 0, bad = 0, len = 0, room = 0;
    if (e < n) {
        s = src[e];
        d = dst[e];
        bad = s < 0 || s >= c.B || d < 0 || d >= c.B;
        if (!bad) {
            len = c.lens[s];
            room = c.room[s];
            mark(is_src, s);
            bad = mark(is_dst, d) || c.lens[d] != 0 || len < 0 || len > c.maxctx;
        }
    }
    __syncthreads();
    if (e < n && !bad) bad = is_src[d >> 5] >> (d & 31) & 1;
    int total;
    const int part = e < n && !bad ? len % c.ps : 0;
    int from = -1, wfrom = -1;           // the partly filled pages
    if (part) {
        const size_t at = (size_t)s * c.width + len / c.ps;
        from = c.table[at];
        if (c.nw) wfrom = c.wtable[at];
    }
    const int rank = block_scan(part > 0, &total);
    if (part > 0) { entry_of[rank] = e; dst_of[e] = d; at_of[e] = len / c.ps; }
    int refused = __syncthreads_or(bad) ? kPagedBadEntry : 0;
    if (!refused && total > 0) { pages.count(); wpages.count(); }
    if (!refused && total > 0 && (pages.total < total || (c.nw && wpages.total < total))) refused = kPagedNoPages;
    if (e == 0) {
        c.scratch[0] = refused ? 0 : n;
        if (refused) atomicOr(c.flag, refused);
    }
    if (refused) return;
    int32_t *const move = c.scratch + 8;
    if (e < n) {
        move[4 * e + 0] = from;
        move[4 * e + 2] = wfrom;
        move[4 * e + 1] = move[4 * e + 3] = -1;
    }
    __syncthreads();
    auto give = [&](int r, int page, int32_t *table, int32_t *refs, int which) {
        const int x = entry_of[r];
        table[(size_t)dst_of[x] * c.width + at_of[x]] = page;
        refs[page] = 1;
        move[4 * x + which] = page;
    };
    if (total > 0) {
        pages.take(total, [&](int r, int page) { give(r, page, c.table, c.refs, 1); });
        if (c.nw) wpages.take(total, [&](int r, int page) { give(r, page, c.wtable, c.wrefs, 3); });
    }
    if (e < n) { c.lens[d] = len; c.room[d] = room; }
}

// blockIdx.y: entry; blockIdx.x: 0 the tables, then one stream each (key, value, window)
__global__ __launch_bounds__(256) void paged_fork_copy_kernel(pod_paged_view c, const int32_t *src, const int32_t *dst)
{
    const int e = blockIdx.y;
    if (e >= c.scratch[0]) return;
    const int s = src[e], d = dst[e], len = c.lens[s];
    if (blockIdx.x == 0) {
        for (int i = threadIdx.x; i < len / c.ps; i += 256) {
            const int page = c.table[(size_t)s * c.width + i], wpage = c.nw ? c.wtable[(size_t)s * c.width + i] : -1;
            c.table[(size_t)d * c.width + i] = page;
            if (page >= 0 && page < c.np) atomicAdd(c.refs + page, 1);
            if (c.nw) c.wtable[(size_t)d * c.width + i] = wpage;
            if (wpage >= 0 && wpage < c.nw) atomicAdd(c.wrefs + wpage, 1);
        }
        return;
    }
    const int part = len % c.ps;
    if (part == 0) return;
    int stream = blockIdx.x - 1;
    const bool window = stream >= c.kstreams + c.vstreams;
    const int32_t *const move = c.scratch + 8 + 4 * e + (window ? 2 : 0);
    const int from = move[0], to = move[1], pages = window ? c.nw : c.np;
    if (from < 0 || from >= pages || to < 0) return;
    size_t off = c.off_keys;
    if (window) { stream -= c.kstreams + c.vstreams; off = c.off_wkeys; }
    else if (stream >= c.kstreams) { stream -= c.kstreams; off = c.off_values; }
    const size_t page_bytes = (size_t)c.ps * c.D * 2;
    char *const b = c.base + off + (size_t)stream * pages * page_bytes;
    const pod_u32x4 *const x = (const pod_u32x4 *)(b + from * page_bytes);
    pod_u32x4 *const y = (pod_u32x4 *)(b + to * page_bytes);
    for (int i = threadIdx.x; i < part * (c.D / 8); i += 256) y[i] = x[i];
}

// ---- free

__global__ __launch_bounds__(256) void paged_free_kernel(pod_paged_view c, const int32_t *slots)
{
    const int s = slots[blockIdx.x];
    if (s < 0 || s >= c.B) {
        if (threadIdx.x == 0) atomicOr(c.flag, kPagedBadEntry);
        return;
    }
    // (a slot named twice: each entry is given back by whoever exchanges it first, whatever the other has read)
    const int len = __hip_atomic_load(c.lens + s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const int held = min(max(len, 0) / c.ps + 1, c.width);
    for (int i = threadIdx.x; i < held; i += 256) {
        const int page = atomicExch(c.table + (size_t)s * c.width + i, -1);
        if (page >= 0 && page < c.np) atomicSub(c.refs + page, 1);
        if (c.nw) {
            const int wpage = atomicExch(c.wtable + (size_t)s * c.width + i, -1);
            if (wpage >= 0 && wpage < c.nw) atomicSub(c.wrefs + wpage, 1);
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) { c.lens[s] = 0; c.room[s] = kPagedAnyRoom; }
}

// ---- compact.  scratch: [0] context moves, [1] window moves, [2], [3] pages in use; from 8 on np entries: the r-th move's page from at
// r; then np: where page p >= pages in use goes, at np + p, ... as many for window pages behind

__device__ __forceinline__ int pack_pool(int32_t *refs, int np, int32_t *from, int32_t *to, int *live_out)
{
    constexpr int kPiece = kPieceBits * kBook;
    auto used = [&](int base) { return read_piece(refs, np, base, [](int, int r) { return r > 0; }); };
    const page_piece one = used(0);      // (the only one, mostly: read once)
    auto below = [&](const page_piece &p, int limit) { // bits of the thread's pages below `limit`
        const int n = limit - p.first;
        return n <= 0 ? 0u : n >= p.per ? ~0u >> (32 - p.per) : (1u << n) - 1;
    };
    int mine = __popc(one.bits), live;
    for (int base = kPiece; base < np; base += kPiece) mine += __popc(used(base).bits);
    block_scan(mine, &live);
    int moves = 0;
    for (int base = live / kPiece * kPiece; base < np; base += kPiece) {
        const page_piece p = base ? used(base) : one;
        const unsigned high = p.bits & ~below(p, live);
        int found, at = moves + block_scan(__popc(high), &found);
        for (unsigned b = high; b; b &= b - 1) from[at++] = p.first + __ffs(b) - 1;
        moves += found;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    for (int base = 0, done = 0; base < live; base += kPiece) {
        const page_piece p = base ? used(base) : one;
        const unsigned holes = ~p.bits & below(p, min(live, np));
        int found, at = done + block_scan(__popc(holes), &found);
        for (unsigned b = holes; b && at < moves; b &= b - 1, ++at) {
            const int i = p.first + __ffs(b) - 1, page = from[at];
            refs[i] = refs[page];
            refs[page] = 0;
            to[page] = i;
        }
        done += found;
    }
    *live_out = live;
    return moves;
}

__global__ __launch_bounds__(kBook) void paged_compact_plan_kernel(pod_paged_view c)
{
    int32_t *const from = c.scratch + 8, *const to = from + c.np, *const wfrom = to + c.np, *const wto = wfrom + c.nw;
    const bool window = blockIdx.x; // a workgroup per pool
    int live = 0, moves = 0;
    if (!window) moves = pack_pool(c.refs, c.np, from, to, &live);
    else if (c.nw) moves = pack_pool(c.wrefs, c.nw, wfrom, wto, &live);
    if (threadIdx.x == 0) { c.scratch[window] = moves; c.scratch[2 + window] = live; }
}

__global__ __launch_bounds__(256) void paged_compact_copy_kernel(pod_paged_view c)
{
    const int32_t *const from = c.scratch + 8, *const to = from + c.np, *const wfrom = to + c.np, *const wto = wfrom + c.nw;
    const int moves = c.scratch[0], wmoves = c.scratch[1], live = c.scratch[2], wlive = c.scratch[3];
    for (int s = blockIdx.x; s < c.B; s += gridDim.x) {
        const int held = min((max(c.lens[s], 0) + c.ps - 1) / c.ps, c.width);
        for (int i = threadIdx.x; i < held; i += 256) {
            const size_t at = (size_t)s * c.width + i;
            const int p = c.table[at];
            if (p >= live && p < c.np) c.table[at] = to[p];
            if (c.nw) {
                const int w = c.wtable[at];
                if (w >= wlive && w < c.nw) c.wtable[at] = wto[w];
            }
        }
    }
    const size_t page_bytes = (size_t)c.ps * c.D * 2;
    const int streams = c.kstreams + c.vstreams, pieces = (int)(page_bytes / 16);
    const int64_t items = (int64_t)moves * streams + (int64_t)wmoves * c.wstreams;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const bool window = item >= (int64_t)moves * streams;
        const int64_t it = window ? item - (int64_t)moves * streams : item;
        int stream = (int)(it / (window ? wmoves : moves));
        const int r = (int)(it - (int64_t)stream * (window ? wmoves : moves));
        const int p = window ? wfrom[r] : from[r], t = window ? wto[p] : to[p], pages = window ? c.nw : c.np;
        size_t off = window ? c.off_wkeys : c.off_keys;
        if (!window && stream >= c.kstreams) { stream -= c.kstreams; off = c.off_values; }
        char *const b = c.base + off + (size_t)stream * pages * page_bytes;
        const pod_u32x4 *const x = (const pod_u32x4 *)(b + p * page_bytes);
        pod_u32x4 *const y = (pod_u32x4 *)(b + t * page_bytes);
        for (int i = threadIdx.x; i < pieces; i += 256) y[i] = x[i];
    }
}

// ---- plan of a packed batch

__global__ __launch_bounds__(kBook) void paged_plan_kernel(pod_paged_view c, const int32_t *cu, const int32_t *slots, int n, int rows, pod_paged_plan_view p)
{
    __shared__ unsigned seen[kPagedMaxBatch / 32];
    __shared__ int before[kBook + 1], row0[kBook + 1], count[kBook], longest;
    const int e = threadIdx.x;
    if (e < kPagedMaxBatch / 32) seen[e] = 0;
    __syncthreads();
    int bad = 0, lo = rows, hi = rows, slot = 0, len = 0;
    if (e < n) {
        slot = slots ? slots[e] : e;
        lo = cu[e];
        hi = cu[e + 1];
        bad = slot < 0 || slot >= c.B || lo < 0 || hi < lo || hi > rows || (e == 0 && lo != 0) || (e == n - 1 && hi != rows);
        if (!bad) {
            const int held = c.lens[slot], room = c.room[slot]; // (both under way at once)
            len = held;
            bad = mark(seen, slot) || len < hi - lo || len > c.maxctx || room < hi - lo;
        }
        if (c.nw && !bad && hi > lo) {
            // What the rows attend by their own layers' keys starts at the first row's window (sink pages never go back).  Pages go back oldest
            // first, so the rest is there if that window's first page behind the sink is.
            const int shift = 31 - __clz(c.ps), first = len - (hi - lo), page = max((c.S + c.ps - 1) >> shift, max(first - c.W + 1, 0) >> shift);
            bad = page <= (len - 1) >> shift && c.wtable[(size_t)slot * c.width + page] < 0;
        }
    }
    const bool refused = __syncthreads_or(bad) || n == 0;
    if (e == 0) {
        p.head->valid = 0;
        if (refused && n > 0) atomicOr(c.flag, kPagedBadPlan);
    }
    if (refused) return;
    const int tokens = pod_paged_tile_tokens(c.rep), tiles = e < n ? (hi - lo + tokens - 1) / tokens : 0;
    int total;
    before[e] = block_scan(tiles, &total);
    row0[e] = lo;
    if (e == 0) { before[kBook] = total; row0[kBook] = rows; }
    if (e < n) p.seq[e] = pod_paged_seq{slot, len, len - (hi - lo), lo};
    __syncthreads();
    // The tiles, those with most keys before them first: sorted by counting into at most kBook classes of their last position.
    if (e == 0) longest = 0;
    count[e] = 0;
    __syncthreads();
    atomicMax(&longest, len);
    __syncthreads();
    const int shift = max(32 - __clz(longest) - 10, 0); // longest >> shift < kBook
    auto tile_at = [&](int t) { // tile t of the list by sequences; the sequence x has before[x] <= t < before[x + 1]
        int a = 0, b = kBook;
        while (b - a > 1) {
            const int m = (a + b) / 2;
            if (before[m] <= t) a = m;
            else b = m;
        }
        return pod_paged_tile{a, (t - before[a]) * tokens};
    };
    auto class_of = [&](pod_paged_tile t) {
        const pod_paged_seq s = p.seq[t.seq];
        return kBook - 1 - (min(s.first + t.token + tokens, s.len) >> shift);
    };
    for (int t = e; t < total; t += kBook) atomicAdd(&count[class_of(tile_at(t))], 1);
    __syncthreads();
    int all;
    const int start = block_scan(count[e], &all);
    count[e] = start;
    __syncthreads();
    for (int t = e; t < total; t += kBook) {
        const pod_paged_tile x = tile_at(t);
        p.tile[atomicAdd(&count[class_of(x)], 1)] = x; // (the order inside a class changes no result)
    }
    for (int r = e; r < rows; r += kBook) {
        int a = 0, b = kBook;
        while (b - a > 1) {
            const int m = (a + b) / 2;
            if (row0[m] <= r) a = m;
            else b = m;
        }
        const pod_paged_seq s = p.seq[a];
        p.row[r] = pod_paged_row{s.slot, s.first + (r - s.row0)};
    }
    if (e == 0) { p.head->ntiles = total; p.head->n = n; p.head->rows = rows; p.head->valid = kPagedPlanValid; }
}

// ---- rows into pages: one 16-byte piece of a key row and of a value row per thread

struct store_params {
    pod_paged_view c;
    pod_paged_plan_view p;
    const pod_bf16 *k, *v;
    int64_t ks, vs;
    int n, rows, layer;
    pod_paged_heads heads;
};

__global__ __launch_bounds__(256) void paged_store_kernel(store_params a)
{
    const pod_paged_view &c = a.c;
    if (a.p.head->valid != kPagedPlanValid || a.p.head->n != a.n || a.p.head->rows != a.rows) {
        if (blockIdx.x == 0 && threadIdx.x == 0) atomicOr(c.flag, kPagedBadPlan);
        return;
    }
    const int cpr = c.D / 8, per_row = c.Hkv * cpr;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int row = (int)(i / per_row), x = (int)(i - (int64_t)row * per_row), h = x / cpr, piece = x - h * cpr;
    if (row >= a.rows) return;
    const pod_paged_row to = a.p.row[row];
    if (to.slot < 0 || to.slot >= c.B || to.pos < 0 || to.pos >= c.maxctx) return;
    const pod_u32x4 k = *(const pod_u32x4 *)(a.k + row * a.ks + h * c.D + 8 * piece), v = *(const pod_u32x4 *)(a.v + row * a.vs + h * c.D + 8 * piece);
    const size_t entry = (size_t)to.slot * c.width + to.pos / c.ps;
    const int at = to.pos % c.ps, page = c.table[entry], wpage = a.heads.window[h] >= 0 ? c.wtable[entry] : -1;
    const size_t row_bytes = (size_t)c.D * 2, page_bytes = c.ps * row_bytes;
    if (page >= 0 && page < c.np) {
        *(pod_u32x4 *)(c.base + c.off_values + ((size_t)(a.layer * c.Hkv + h) * c.np + page) * page_bytes + at * row_bytes + 16 * piece) = v;
        if (a.heads.window[h] < 0) *(pod_u32x4 *)(c.base + c.off_keys + ((size_t)a.heads.key[h] * c.np + page) * page_bytes + at * row_bytes + 16 * piece) = k;
    }
    if (wpage >= 0 && wpage < c.nw)
        *(pod_u32x4 *)(c.base + c.off_wkeys + ((size_t)a.heads.window[h] * c.nw + wpage) * page_bytes + at * row_bytes + 16 * piece) = k;
}

} // namespace

int pod_launch_paged_reset(const pod_paged *c, hipStream_t st)
{
    paged_reset_kernel<<<256, 256, 0, st>>>(c->v);
    POD_HIP_TRY(hipGetLastError());
    return POD_OK;
}

int pod_launch_paged_clear(const pod_paged *c, hipStream_t st)
{
    paged_clear_kernel<<<1, kBook, 0, st>>>(c->v);
    POD_HIP_TRY(hipGetLastError());
    return POD_OK;
}

int pod_launch_paged_extend(const pod_paged *c, const int32_t *counts, const int32_t *slots, int n, hipStream_t st)
{
    paged_extend_kernel<<<1, kBook, 0, st>>>(c->v, counts, slots, n);
    POD_HIP_TRY(hipGetLastError());
    return POD_OK;
}

int pod_launch_paged_fork(const pod_paged *c, const int32_t *src, const int32_t *dst, int n, hipStream_t st)
{
    paged_fork_plan_kernel<<<1, kBook, 0, st>>>(c->v, src, dst, n);
    POD_HIP_TRY(hipGetLastError());
    paged_fork_copy_kernel<<<dim3(1 + c->v.kstreams + c->v.vstreams + c->v.wstreams, n), 256, 0, st>>>(c->v, src, dst);
    POD_HIP_TRY(hipGetLastError());
    return POD_OK;
}

int pod_launch_paged_free(const pod_paged *c, const int32_t *slots, int n, hipStream_t st)
{
    paged_free_kernel<<<n, 256, 0, st>>>(c->v, slots);
    POD_HIP_TRY(hipGetLastError());
    return POD_OK;
}

int pod_launch_paged_compact(const pod_paged *c, hipStream_t st)
{
    paged_compact_plan_kernel<<<2, kBook, 0, st>>>(c->v);
    POD_HIP_TRY(hipGetLastError());
    paged_compact_copy_kernel<<<8 * c->cus, 256, 0, st>>>(c->v);
    POD_HIP_TRY(hipGetLastError());
    return POD_OK;
}

int pod_launch_paged_plan(const pod_paged *c, const int32_t *cu, const int32_t *slots, int n, int rows, void *plan, hipStream_t st)
{
    paged_plan_kernel<<<1, kBook, 0, st>>>(c->v, cu, slots, n, rows, pod_paged_plan_at(plan, c->v.rep, n, rows, nullptr));
    POD_HIP_TRY(hipGetLastError());
    return POD_OK;
}

int pod_launch_paged_store(const pod_paged *c, int layer, const void *k, int64_t ks, const void *v, int64_t vs, int n, int rows,
                           const void *plan, hipStream_t st)
{
    store_params a;
    a.c = c->v;
    a.p = pod_paged_plan_at(plan, c->v.rep, n, rows, nullptr);
    a.k = (const pod_bf16 *)k; a.v = (const pod_bf16 *)v; a.ks = ks; a.vs = vs;
    a.n = n; a.rows = rows; a.layer = layer;
    a.heads = pod_paged_make_heads(c, layer);
    const int64_t pieces = (int64_t)rows * c->v.Hkv * (c->v.D / 8);
    if ((pieces + 255) / 256 > 0x7fffffff) return pod_fail(POD_ERR_CAPACITY, "%d rows in one call are too many", rows);
    paged_store_kernel<<<(unsigned)((pieces + 255) / 256), 256, 0, st>>>(a);
    POD_HIP_TRY(hipGetLastError());
    return POD_OK;
}
