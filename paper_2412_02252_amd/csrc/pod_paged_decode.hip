// One token per sequence over the paged cache: split over the length, joined inside the launch.
//
// Eq. 3 of the paper at the last position of each sequence, one softmax.  The launch streams every key and value row once, so HBM bounds
// it; the design keeps loads in flight and every compute unit busy to the end whatever the lengths are:
//  - The rows of all (sequence, kv head) pairs are one list of 32-token tiles, and every workgroup of one resident round takes a run of it,
//    equal to a tile, or one that ends with its pair (kBorder); its four waves take tiles in turn.  Lengths and tables are read on the device, nothing depends on the host.
//  - A pair that a workgroup holds whole is finished there.  The parts of the others (maximum, sum, sum of values) go through memory to
//    whichever of the pair's workgroups arrives last, which adds them in the order of the list: the result does not depend on who it is.
//  - The query heads of a kv head are the 16 columns of the products (S^T = K Q^T, O^T += V^T P, v_mfma_f32_16x16x32): head = lane % 16 in
//    both, so a lane keeps one head's maximum and sum, and its probabilities are already the second product's operand.  K rows are loaded whole
//    (one request = four rows of 256 bytes) and turned through a piece of LDS of the wave; V is turned in registers (v_perm_b32).
//  - The new token's row is read from the call's arguments by the wave that has the last tile, and stored by it: no wait in between.
// 16 sequences of 4096 .. 32768 tokens x 8 kv heads x 128 (1087 MB): 179 us, 6.1 TB/s; one of 32768 (134 MB): 33 us; 32 of 300 .. 4096 x 4 x 64 (47 MB): 17.8.
// Weights are rounded to the type for the second product, whose operands have 16 bits (error against 64 bits 1.2 to 1.4 times that of rounding the result alone); the
// sum that divides them, the maximum and all sums of products keep 32.
// At an upper layer the list of a pair is its distant tiles (the lowest layer's keys and query), then the sink and window tiles (own keys,
// window pages); a tile with both kinds is in both parts, each masking what is the other's.
#include "pod_paged.h"
#include "pod_paged_device.h"

namespace {

constexpr int kWaves = 4, kTile = 32;
constexpr int kMinRun = kWaves; // tiles of a run at least, while there are that many
// A run over a pair's border ends with two pairs' sums to hand over, one after the other, some 4 us that weigh as much as this many tiles: pairs
// get runs of their own where the longest such run is no more than that above the average.  (32 chats x 4 heads x 64, 11 tiles on average
// against 15: 21.8 us over borders, 18.0 with own runs; 16 documents x 8 x 128, 130 against 173: 181 and 183; 1 x 2 x 64 x 2048: 14.3 and 10.4.)
constexpr unsigned kBorder = 8;
constexpr int kMaxWgs = 512; // workgroups of a launch, and so the parts of a pair, at most

struct decode_params {
    pod_paged_view c;
    const int32_t *slots;
    const char *q, *qs, *k, *v;                     // rows of 16-bit elements
    int64_t q_stride, qs_stride, k_stride, v_stride; // bytes
    char *out;
    float *part, *part_ml;                          // [2 * workgroups][rep][D], [2 * workgroups][rep][2]: a run ends one pair and begins another
    int n, layer, low_heads;                        // low_heads: kv heads without keys in window pages
    float scale_log2e;
    pod_paged_heads heads;
};

// Tiles of a pair with n tokens in walking order: nd distant ones from d0, np1 sink tiles from 0, window tiles from wb.
struct tiles { int d0, nd, np1, wb, count; };
__device__ inline tiles tiles_of(int n, int S, int W, bool low)
{
    tiles t = {0, 0, 0, 0, 0};
    const int last = n - 1;
    if (!low) {
        if (last - W >= S) { t.d0 = S / kTile; t.nd = (last - W) / kTile - t.d0 + 1; }
        if (S > 0) t.np1 = (min(S, n) - 1) / kTile + 1;
        t.wb = max(t.np1, last - W + 1 > 0 ? (last - W + 1) / kTile : 0);
    }
    t.count = t.nd + t.np1 + max(last / kTile - t.wb + 1, 0);
    return t;
}
__device__ inline int count_of(int n, int S, int W, bool low) { return n > 0 ? tiles_of(n, S, W, low).count : 0; }

// Parts travel between workgroups on any XCD, whose L2s are not coherent: stores and loads that go through to memory.
__device__ inline void store_part(float *p, float v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
// Read 16 bytes at a time past this compute unit's L1 and this XCD's L2 (sc1).
constexpr int kRawBuffer = 0x00020000, kBufferSC1 = 16;

// The parts of workgroups first .. first + parts - 1 added up, in that order whoever does it, by one workgroup: the weights of the parts first
// (a wave per head), then the rows, every load of a thread in flight before the first is used.  Groups of D / 4 lanes take a row each,
// as many groups to a head as there are.
template <class T, int D>
__device__ __forceinline__ void merge_parts(const decode_params &p, char *lds, int first, int parts, char *out)
{
    constexpr int LPR = D / 4, NG = kWaves * 64 / LPR, UN = 8; // lanes a row, rows at a time, rows of a thread in flight
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, rep = p.c.rep;
    const __amdgpu_buffer_rsrc_t rows = __builtin_amdgcn_make_buffer_rsrc((void *)p.part, 0, 2 * kMaxWgs * rep * D * 4, kRawBuffer);
    const __amdgpu_buffer_rsrc_t mls = __builtin_amdgcn_make_buffer_rsrc((void *)p.part_ml, 0, 2 * kMaxWgs * rep * 8, kRawBuffer);
    auto slot_of = [&](int i) { return (unsigned)(2 * (first + i) + (i == 0)); }; // (the first one starts at the pair's first tile)
    float *const w = (float *)lds;                        // [rep][parts]
    f32x4 *const sums = (f32x4 *)(w + (rep * parts + 3) / 4 * 4); // [NG][LPR]
    for (int head = wave; head < rep; head += kWaves) {
        float M = kLowestLogit, l = 0.f;
        for (int i = lane; i < parts; i += 64) {
            const f32x2 ml = __builtin_bit_cast(f32x2, __builtin_amdgcn_raw_buffer_load_b64(mls, (slot_of(i) * rep + head) * 8, 0, kBufferSC1));
            const float m = ml.x, now = fmaxf(M, m);
            l = l * __builtin_amdgcn_exp2f(M - now) + ml.y * __builtin_amdgcn_exp2f(m - now);
            M = now;
            w[head * parts + i] = m;
        }
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) {
            const float m = __shfl_xor(M, off), other = __shfl_xor(l, off), now = fmaxf(M, m);
            l = l * __builtin_amdgcn_exp2f(M - now) + other * __builtin_amdgcn_exp2f(m - now);
            M = now;
        }
        const float inv = 1.f / __shfl(l, 0);
        M = __shfl(M, 0);
        for (int i = lane; i < parts; i += 64) w[head * parts + i] = __builtin_amdgcn_exp2f(w[head * parts + i] - M) * inv;
    }
    __syncthreads();
    const int g = tid / LPR, x = tid % LPR, per_head = max(NG / rep, 1), share = g % per_head;
    for (int h0 = 0; h0 < rep; h0 += NG / per_head) {
        const int head = h0 + g / per_head;
        f32x4 a = {0.f, 0.f, 0.f, 0.f};
        if (head < rep)
            for (int i0 = share; i0 < parts; i0 += UN * per_head) {
                f32x4 r[UN];
#pragma unroll
                for (int k = 0; k < UN; ++k) {
                    const int i = min(i0 + k * per_head, parts - 1);
                    r[k] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rows, ((slot_of(i) * rep + head) * D + 4 * x) * 4, 0, kBufferSC1));
                }
#pragma unroll
                for (int k = 0; k < UN; ++k)
                    if (i0 + k * per_head < parts) a += r[k] * w[head * parts + i0 + k * per_head];
            }
        sums[g * LPR + x] = a;
        __syncthreads();
        if (share == 0 && head < rep) {
            for (int k = 1; k < per_head; ++k) a += sums[(g + k) * LPR + x];
            *(u32x2 *)(out + (size_t)head * D * 2 + 8 * x) = u32x2{T::pack(a[0], a[1]), T::pack(a[2], a[3])};
        }
        __syncthreads();
    }
}

template <class T, int D>
__global__ __launch_bounds__(kWaves * 64, 2) void paged_decode_kernel(decode_params p)
{
    constexpr int CPR = D / 8, RPI = 64 / CPR, NLD = kTile / RPI, KST = D / 32, RB = D * 2; // pieces a row, rows a K request, K requests a tile
    constexpr int VD = D / 16;          // dims of a token's value row that a lane loads
    constexpr int RS = D + 4 * (D / 32) + 1;  // row stride of the merge buffer: 16 heads' rows in different banks
    typedef typename vec_of<VD / 2>::type vpiece;
    constexpr size_t kTileBytes = (size_t)kWaves * kTile * RB, kWaveSums = sizeof(float) * kWaves * 16 * RS, kWeights = (16 * kMaxWgs + 4 * kWaves * 64) * sizeof(float);
    __shared__ __attribute__((aligned(16))) char lds[kTileBytes > kWaveSums ? (kTileBytes > kWeights ? kTileBytes : kWeights) : (kWaveSums > kWeights ? kWaveSums : kWeights)];
    __shared__ float sm_m[kWaves][16], sm_l[kWaves][16];
    __shared__ int cum[kPagedMaxBatch], sums[kWaves], sm_last;

    const pod_paged_view &c = p.c;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), m16 = lane & 15, j = lane >> 4;
    const int S = c.S, W = c.W, rep = c.rep, hkv = c.Hkv;
    // The arguments lie on several cache lines; without this they are fetched one after the other, each where it is first used.
    asm volatile("" ::"s"(p.slots), "s"(c.lens), "s"(c.room), "s"(c.table), "s"(c.B), "s"(c.maxctx), "s"(S), "s"(W), "s"(hkv), "s"(p.n), "s"(p.low_heads), "s"(p.k_stride), "s"(p.part), "s"(p.heads.window[0]));

    // ---- the list: tiles up to and with each sequence's.  Of up to 64 sequences every wave keeps them in a lane each, without a barrier; more
    // are summed up in LDS.
    const bool few = p.n <= 64;
    auto units_of_all = [&](int n, int unit) __attribute__((always_inline)) { // pieces of `unit` tiles of all heads of a sequence
        const int low = p.low_heads ? (unsigned)(count_of(n, S, W, true) + unit - 1) / (unsigned)unit : 0, up = p.low_heads < hkv ? (unsigned)(count_of(n, S, W, false) + unit - 1) / (unsigned)unit : 0;
        return p.low_heads * low + (hkv - p.low_heads) * up;
    };
    auto read_entry = [&](int e, int &slot, int &n) __attribute__((always_inline)) { // slot and tokens of an entry; the tiles of all its heads
        slot = p.slots ? p.slots[e] : e;
        const bool bad = slot < 0 || slot >= c.B;
        if (bad && blockIdx.x == 0) atomicOr(c.flag, kPagedBadEntry);
        const int at = bad ? 0 : slot, held = c.lens[at], room = c.room[at]; // (both under way at once)
        n = bad || (p.k && room < 1) ? 0 : held; // (room for the new token was refused: the last token is another one)
        if (n < 0 || n > c.maxctx) n = 0;
        return p.low_heads * (p.low_heads ? count_of(n, S, W, true) : 0) + (hkv - p.low_heads) * (p.low_heads < hkv ? count_of(n, S, W, false) : 0);
    };
    auto lane_scan = [&](int x) __attribute__((always_inline)) { // sum of the lanes up to and with this one
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int y = __shfl_up(x, off);
            if (lane >= off) x += y;
        }
        return x;
    };
    int my_slot = 0, my_n = 0, my_cum = 0, total, unit = 1; // (from here on lengths are in pieces of `unit` tiles)
    bool own = false;                                 // no run holds tiles of two pairs
    if (few) {
        if (lane < p.n) my_cum = read_entry(lane, my_slot, my_n);
        if (p.n > 1) my_cum = lane_scan(my_cum);
        total = __builtin_amdgcn_readlane(my_cum, p.n - 1);
        // Runs of `unit` tiles that end where their pair does: sum of ceil(tiles / unit) over the pairs <= total / unit + pairs.
        const int room = (int)gridDim.x - p.n * hkv;
        if (room > 0) {
            const unsigned longest = (unsigned)(total + room - 1) / (unsigned)room;
            own = (uint64_t)longest * gridDim.x <= (uint64_t)(unsigned)total + kBorder * gridDim.x;
            if (own) {
                unit = max((int)longest, kMinRun);
                my_cum = lane < p.n ? units_of_all(my_n, unit) : 0;
                if (p.n > 1) my_cum = lane_scan(my_cum);
                total = __builtin_amdgcn_readlane(my_cum, p.n - 1);
            }
        }
    } else {
        int before = 0;
        for (int base = 0; base < p.n; base += kWaves * 64) {
            const int e = base + tid;
            int slot, n;
            const int incl = lane_scan(e < p.n ? read_entry(e, slot, n) : 0);
            if (lane == 63) sums[wave] = incl;
            __syncthreads();
            int ahead = before;
            for (int w = 0; w < kWaves; ++w) {
                if (w < wave) ahead += sums[w];
                before += sums[w];
            }
            if (e < p.n) cum[e] = ahead + incl;
            __syncthreads();
        }
        total = __builtin_amdgcn_readfirstlane(before);
    }
    auto cum_at = [&](int e) __attribute__((always_inline)) { // pieces before entry e's
        return e == 0 ? 0 : few ? __builtin_amdgcn_readlane(my_cum, e - 1) : __builtin_amdgcn_readfirstlane(cum[e - 1]);
    };
    for (int e = blockIdx.x; e < p.n; e += gridDim.x) // entries without a token
        if (cum_at(e + 1) == cum_at(e))
            for (int i = tid; i < c.Hq * D / 2; i += kWaves * 64) ((unsigned *)p.out)[(size_t)e * (c.Hq * D / 2) + i] = 0;
    // `runs` workgroups have one: `longer` of run + 1 pieces, then the others of run
    unsigned runs = total, run = 1, longer = 0;
    if (!own) {
        runs = min(gridDim.x, (unsigned)(total + kMinRun - 1) / kMinRun);
        if (blockIdx.x < runs) { run = (unsigned)total / runs; longer = (unsigned)total - run * runs; }
    }
    if (blockIdx.x >= runs) return;
    const unsigned border = longer * (run + 1);
    auto start_of = [&](unsigned w) __attribute__((always_inline)) { return (int)(w * run + min(w, longer)); };
    auto run_of = [&](unsigned at) __attribute__((always_inline)) { return own ? (int)at : (int)(at < border ? at / (run + 1) : longer + (at - border) / run); }; // whose piece it is
    int u = __builtin_amdgcn_readfirstlane(start_of(blockIdx.x));
    const int u_end = __builtin_amdgcn_readfirstlane(start_of(blockIdx.x + 1));
    int e = 0; // the entry of piece u
    if (few) e = __popcll(__ballot(lane < p.n && my_cum <= u));
    else
        for (int hi = p.n; hi - e > 1;) { // cum_at(e) <= u < cum_at(hi)
            const int mid = (e + hi) / 2;
            if (cum[mid - 1] <= u) e = mid;
            else hi = mid;
        }
    e = __builtin_amdgcn_readfirstlane(e);

    u32x4 *const ldsK = (u32x4 *)lds + (size_t)wave * kTile * CPR;
    const int kr = lane / CPR, kc = lane % CPR;

    while (u < u_end) {
        while (cum_at(e + 1) <= u) ++e;
        // ---- the pair and its part: pieces r0 .. r1 - 1 of `per`, tiles first_tile .. t_end - 1
        const int slot = few ? __builtin_amdgcn_readlane(my_slot, e) : __builtin_amdgcn_readfirstlane(p.slots ? p.slots[e] : e);
        const int n = few ? __builtin_amdgcn_readlane(my_n, e) : __builtin_amdgcn_readfirstlane(c.lens[slot]);
        auto pieces = [&](bool low) __attribute__((always_inline)) { // of a pair
            const unsigned count = count_of(n, S, W, low);
            return (int)(own ? (count + unit - 1) / (unsigned)unit : count);
        };
        int h = 0, r0 = u - cum_at(e), per;
        if (p.low_heads == hkv || p.low_heads == 0) {
            per = pieces(p.low_heads != 0);
            h = (unsigned)r0 / (unsigned)per;
            r0 -= h * per;
        } else {
            const int per_low = pieces(true), per_up = pieces(false);
            for (;; ++h) {
                per = p.heads.window[h] < 0 ? per_low : per_up;
                if (r0 < per) break;
                r0 -= per;
            }
        }
        const int pair_u0 = u - r0, r1 = min(per, r0 + u_end - u);
        h = __builtin_amdgcn_readfirstlane(h);
        const int wstream = p.heads.window[h];
        const bool low = p.low_heads == hkv || (p.low_heads > 0 && wstream < 0); // (the same; where one answer serves all heads it need not wait for the table)
        const tiles tl = tiles_of(n, S, W, low);
        const int first_tile = __builtin_amdgcn_readfirstlane(r0 * unit), t_end = __builtin_amdgcn_readfirstlane(min(r1 * unit, tl.count));
        const int ndist = low ? 0 : max(n - W - S, 0); // tokens S .. S + ndist - 1 are distant

        const size_t page_bytes = (size_t)c.ps * RB;
        const gbytes kpool = (gbytes)(c.base + c.off_keys) + (size_t)p.heads.key[h] * c.np * page_bytes;
        const gbytes wpool = low ? kpool : (gbytes)(c.base + c.off_wkeys) + (size_t)wstream * c.nw * page_bytes;
        const gbytes vpool = (gbytes)(c.base + c.off_values) + (size_t)(p.layer * hkv + h) * c.np * page_bytes;
        const gints table = (gints)(c.table + (size_t)slot * c.width), wtable = (gints)(c.wtable + (size_t)slot * c.width);
        const int ps_shift = 31 - __builtin_clz(c.ps);

        auto visit = [&](int v, int &t0, bool &dist) { // v-th tile of the list
            dist = v < tl.nd;
            t0 = kTile * (v + (dist ? tl.d0 : v < tl.nd + tl.np1 ? -tl.nd : tl.wb - tl.nd - tl.np1));
        };
        // rows of a tile: two halves of 16 tokens, each inside one page (the last token's page for a half behind the end)
        struct bases { gbytes k[2], v[2]; };
        bool lost = false; // an own key that the token attends lies in a window page that is gone (a refused extend may have given it back)
        auto bases_of = [&](int t0, bool dist) {
            bases b;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int at = min(t0 + 16 * half, n - 1), i = at >> ps_shift;
                int page = table[i], kpage = (dist || low ? table : wtable)[i];
                page = (unsigned)page < (unsigned)c.np ? page : 0;
                if (__builtin_expect((unsigned)kpage >= (unsigned)(dist || low ? c.np : c.nw), 0)) {
                    asm volatile(""); // (keeps this a branch)
                    lost = lost || (!dist && (at < S || at + 15 >= n - W));
                    kpage = 0;       // any page: its keys are masked, or nothing of the pair counts
                }
                const size_t row = (size_t)(at & (c.ps - 1)) * RB;
                b.v[half] = vpool + page * page_bytes + row;
                b.k[half] = (dist ? kpool : wpool) + kpage * page_bytes + row;
            }
            return b;
        };
        const gbytes k_new = p.k ? (gbytes)p.k + e * p.k_stride + h * RB : nullptr, v_new = p.k ? (gbytes)p.v + e * p.v_stride + h * RB : nullptr;
        u32x4 kreg[NLD];
        vpiece vreg[8];
        auto load_tile = [&](int t0, const bases &b) __attribute__((always_inline)) {
            if (__builtin_expect(t0 + kTile < n, 1)) {
#pragma unroll
                for (int i = 0; i < NLD; ++i) {
                    const int half = RPI * i / 16;
                    kreg[i] = *(const gvec)(b.k[half] + (unsigned)((RPI * i - 16 * half + kr) * RB + 16 * kc));
                }
#pragma unroll
                for (int x = 0; x < 8; ++x)
                    vreg[x] = __builtin_nontemporal_load((const __attribute__((address_space(1))) vpiece *)(b.v[x >> 2] + (unsigned)((4 * j + (x & 3)) * RB + 2 * VD * m16)));
            } else { // rows up to the last token, whose row may still be the caller's
#pragma unroll
                for (int i = 0; i < NLD; ++i) {
                    const int half = RPI * i / 16, first = min(t0 + 16 * half, n - 1), at = min(t0 + RPI * i + kr, n - 1);
                    gbytes row = b.k[half] + (unsigned)((at - first) * RB);
                    if (k_new && at == n - 1) row = k_new;
                    kreg[i] = *(const gvec)(row + 16 * kc);
                }
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    const int first = min(t0 + 16 * (x >> 2), n - 1), at = min(t0 + 16 * (x >> 2) + 4 * j + (x & 3), n - 1);
                    gbytes row = b.v[x >> 2] + (unsigned)((at - first) * RB);
                    if (v_new && at == n - 1) row = v_new;
                    vreg[x] = *(const __attribute__((address_space(1))) vpiece *)(row + 2 * VD * m16);
                }
                // The two branches' loads stay apart: merged behind them, whole tiles would pay for the clamped addresses too, and lose their hint.
                asm volatile("" ::: "memory");
            }
        };

        f32x4 acc[VD];
#pragma unroll
        for (int x = 0; x < VD; ++x) acc[x] = f32x4{0.f, 0.f, 0.f, 0.f};
        float m_run = kLowestLogit, l_run = 0.f;
        u32x4 qf[KST];
        auto load_q = [&](bool dist) __attribute__((always_inline)) {
            const gbytes row = (gbytes)(dist ? p.qs : p.q) + e * (dist ? p.qs_stride : p.q_stride) + (h * rep + min(m16, rep - 1)) * RB;
#pragma unroll
            for (int s = 0; s < KST; ++s) qf[s] = *(const gvec)(row + 64 * s + 16 * j);
#pragma unroll
            for (int s = 0; s < KST; ++s) asm volatile("" : "+v"(qf[s])); // awaited here, once or twice a pair, and not before every tile's products
        };

        int v = first_tile + wave;
        int t0 = 0, t0_next = 0;
        bool dist = false, dist_next = false;
        bases next = {};
        if (v < t_end) {
            visit(v, t0, dist);
            const bases b = bases_of(t0, dist);
            load_q(dist);
            load_tile(t0, b);
            if (v + kWaves < t_end) {
                visit(v + kWaves, t0_next, dist_next);
                next = bases_of(t0_next, dist_next);
            }
        }
        for (; v < t_end; v += kWaves) {
#pragma unroll
            for (int i = 0; i < NLD; ++i) {
                const int r = RPI * i + kr;
                ldsK[r * CPR + (kc ^ (r % CPR))] = kreg[i];
            }
            vpiece vcur[8];
#pragma unroll
            for (int x = 0; x < 8; ++x) vcur[x] = vreg[x];
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < KST; ++s) {
                const int col = 4 * s + j;
                s0 = T::mfma16(ldsK[m16 * CPR + (col ^ (m16 % CPR))], qf[s], s0);
                s1 = T::mfma16(ldsK[(16 + m16) * CPR + (col ^ ((16 + m16) % CPR))], qf[s], s1);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            const int t_now = t0;
            const bool dist_now = dist;
            if (v + kWaves < t_end) {
                t0 = t0_next;
                dist = dist_next;
                load_tile(t0, next);
                if (dist != dist_now) load_q(dist);
                if (v + 2 * kWaves < t_end) {
                    visit(v + 2 * kWaves, t0_next, dist_next);
                    next = bases_of(t0_next, dist_next);
                }
            }
            float sc[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) sc[i] = (i < 4 ? s0[i & 3] : s1[i & 3]) * p.scale_log2e;
            // whole tiles count all their tokens
            const bool whole = dist_now ? t_now >= S && t_now + kTile <= S + ndist : t_now + kTile <= n && (ndist == 0 || t_now + kTile <= S || t_now >= S + ndist);
            if (!whole) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int at = t_now + 16 * (i >> 2) + 4 * j + (i & 3);
                    if (at >= n || ((unsigned)(at - S) < (unsigned)ndist) != dist_now) sc[i] = -__builtin_inff();
                }
            }
            float top = fmaxf(fmaxf(fmaxf(sc[0], sc[1]), fmaxf(sc[2], sc[3])), fmaxf(fmaxf(sc[4], sc[5]), fmaxf(sc[6], sc[7])));
            top = max_over_16s(top);
            const float m_new = fmaxf(m_run, top), alpha = __builtin_amdgcn_exp2f(m_run - m_new), shift = m_new - T::spare(0.f);
            float part = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                sc[i] = __builtin_amdgcn_exp2f(sc[i] - shift);
                part += sc[i];
            }
            l_run = l_run * alpha + part;
            m_run = m_new;
            const u32x4 pf = {T::pack(sc[0], sc[1]), T::pack(sc[2], sc[3]), T::pack(sc[4], sc[5]), T::pack(sc[6], sc[7])};
#pragma unroll
            for (int x = 0; x < VD; ++x) {
                const unsigned sel = x & 1 ? 0x07060302u : 0x05040100u; // the odd or the even dim of a pair
                u32x4 vt;
#pragma unroll
                for (int t = 0; t < 4; ++t) vt[t] = __builtin_amdgcn_perm(vcur[2 * t + 1][x >> 1], vcur[2 * t][x >> 1], sel);
                acc[x] = T::mfma16(vt, pf, acc[x] * alpha);
            }
        }
        if (p.k && r1 == per && wave == (tl.count - 1 - first_tile) % kWaves && lane < 2 * CPR) { // the new token's rows, by the wave that has the last tile
            const int at = n - 1, i = at >> ps_shift, page = table[i], kpage = low ? page : wtable[i];
            const size_t row = (size_t)(at & (c.ps - 1)) * RB + 16 * kc;
            typedef __attribute__((address_space(1))) char *gout;
            if (lane < CPR) {
                const u32x4 r = *(const gvec)(k_new + 16 * kc);
                if ((unsigned)kpage < (unsigned)(low ? c.np : c.nw)) *(__attribute__((address_space(1))) u32x4 *)((gout)wpool + kpage * page_bytes + row) = r;
            } else {
                const u32x4 r = *(const gvec)(v_new + 16 * kc);
                if ((unsigned)page < (unsigned)c.np) *(__attribute__((address_space(1))) u32x4 *)((gout)vpool + page * page_bytes + row) = r;
            }
        }

        // ---- the four waves' sums become one.  acc[x][i] is O^T[dim VD (4 j + i) + x][head m16]
        l_run = sum_over_16s(l_run);
        if (lost) { // a maximum above every other, an infinite sum, no values: the entry's row becomes zeros, whoever adds the parts
            if (lane == 0) atomicOr(c.flag, kPagedBadEntry);
            m_run = -kLowestLogit;
            l_run = __builtin_inff();
#pragma unroll
            for (int x = 0; x < VD; ++x) acc[x] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        __syncthreads(); // every wave is done with its K tiles (and with the last pair's merge)
        float *const sm = (float *)lds;
        if (m16 < rep) {
#pragma unroll
            for (int x = 0; x < VD; ++x)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int dim = VD * (4 * j + i) + x;
                    sm[(wave * rep + m16) * RS + dim + 4 * (dim >> 5)] = acc[x][i];
                }
            if (j == 0) { sm_m[wave][m16] = m_run; sm_l[wave][m16] = l_run; }
        }
        __syncthreads();
        const bool done = r0 == 0 && r1 == per;
        const size_t part = 2 * (size_t)blockIdx.x + (r0 == 0);
        for (int t = tid; t < rep * (D / 2); t += kWaves * 64) {
            const int head = t / (D / 2), dim = 2 * (t % (D / 2));
            float M = fmaxf(fmaxf(sm_m[0][head], sm_m[1][head]), fmaxf(sm_m[2][head], sm_m[3][head])), a0 = 0.f, a1 = 0.f, l = 0.f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const float f = __builtin_amdgcn_exp2f(sm_m[w][head] - M);
                const float *const row = sm + (w * rep + head) * RS + dim + 4 * (dim >> 5);
                a0 += f * row[0];
                a1 += f * row[1];
                l += f * sm_l[w][head];
            }
            if (done) {
                const float inv = 1.f / l;
                *(unsigned *)(p.out + ((size_t)e * c.Hq + h * rep + head) * RB + 2 * dim) = T::pack(a0 * inv, a1 * inv);
            } else {
                store_part(p.part + (part * rep + head) * D + dim, a0);
                store_part(p.part + (part * rep + head) * D + dim + 1, a1);
                if (dim == 0) { store_part(p.part_ml + (part * rep + head) * 2, M); store_part(p.part_ml + (part * rep + head) * 2 + 1, l); }
            }
        }
        if (!done) { // workgroups first .. first + parts - 1 have a part of the pair; the last to arrive adds them
            const int first = run_of(pair_u0), parts = run_of(pair_u0 + per - 1) - first + 1;
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); // this thread's part is in memory
            __syncthreads();
            if (tid == 0) {
                const int before = __hip_atomic_fetch_add(c.tickets + (size_t)e * hkv + h, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                sm_last = before == parts - 1;
                if (sm_last) __hip_atomic_store(c.tickets + (size_t)e * hkv + h, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
            __syncthreads();
            if (sm_last) {
                merge_parts<T, D>(p, lds, first, parts, p.out + ((size_t)e * c.Hq + h * rep) * RB);
            }
        }
        u += r1 - r0;
        __syncthreads(); // the merge buffer is free again
    }
}

} // namespace

size_t pod_paged_decode_workspace(const pod_layout &ly) { return (size_t)2 * kMaxWgs * ly.rep * (ly.D + 2) * sizeof(float); }

int pod_launch_paged_decode(const pod_paged *c, const pod_paged_call &a, hipStream_t st)
{
    const pod_paged_view &v = c->v;
    decode_params p;
    p.c = v;
    p.slots = a.slots;
    p.q = (const char *)a.q; p.qs = (const char *)a.qs; p.k = (const char *)a.k; p.v = (const char *)a.v;
    p.q_stride = 2 * a.q_stride; p.qs_stride = 2 * a.qs_stride; p.k_stride = 2 * a.k_stride; p.v_stride = 2 * a.v_stride;
    p.out = (char *)a.out;
    p.part = (float *)a.workspace;
    p.part_ml = p.part + (size_t)2 * kMaxWgs * v.rep * v.D;
    p.n = a.n; p.layer = a.layer;
    p.scale_log2e = a.scale * 1.4426950408889634f;
    p.heads = pod_paged_make_heads(c, a.layer);
    p.low_heads = 0;
    for (int h = 0; h < v.Hkv; ++h) p.low_heads += p.heads.window[h] < 0;
    // one resident round; no more than the longest sequences could use (at most three tiles are in both parts of a pair's list, and
    // entries without a token are cleared by some workgroup)
    const int64_t most = (int64_t)a.n * v.Hkv * ((v.maxctx + kTile - 1) / kTile + 3 + kMinRun - 1) / kMinRun;
    if (most > 0x7fffffff / kMinRun) return pod_fail(POD_ERR_CAPACITY, "%d sequences of up to %d tokens with %d kv heads in one call are too many", a.n, v.maxctx, v.Hkv);
    int wgs = 2 * c->cus < kMaxWgs ? 2 * c->cus : kMaxWgs;
    if (wgs > most) wgs = (int)most;
    void *const fn = v.D == 128 ? (c->dtype == POD_TYPE_FP16 ? (void *)paged_decode_kernel<type_fp16, 128> : (void *)paged_decode_kernel<type_bf16, 128>)
                                : (c->dtype == POD_TYPE_FP16 ? (void *)paged_decode_kernel<type_fp16, 64> : (void *)paged_decode_kernel<type_bf16, 64>);
    void *args[] = {&p};
    POD_HIP_TRY(hipLaunchKernel(fn, dim3((unsigned)wgs), dim3(kWaves * 64), args, 0, st));
    POD_HIP_TRY(hipGetLastError());
    return POD_OK;
}
