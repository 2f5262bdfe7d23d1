// Attention over a paged cache of keys and values, with prefixes that groups of sequences share.
//
// Row t of a sequence with n query rows and L cached tokens of its own sees its group's whole prefix and own tokens
// j <= L - n + t:  out = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m),  s_j = scale q.k_j,  m a running maximum.
//
// Work.  The R = Hq / Hk query heads that share a KV head are rows of one product: row r = t R + (h mod R).  A segment is a
// prefix (with the rows of all its group's sequences) or a sequence's own tokens (with its rows).  An ITEM is one KV head and one
// tile of M rows of a segment; its KV tokens are cut into TILES.  All tiles of all items stand in one line, each item with kCost
// tiles' worth of room before it (what beginning and ending a piece takes; wide tiles, room 1, 2, 3, 4, at 1965 MHz: questions behind
// shared images 376, 296, 276, 296 us, prefill 327, 313, 324, 328), and every worker takes an equal, contiguous share of it: no worker waits
// for another, and one long sequence fills the GPU as well as many short ones.  A prefix is read once per M rows of its whole group.  The lengths are only known on the device; every
// CTA adds them up itself (a launch for it would cost more).
// Joining.  An item that one worker held whole, with nothing else to join, is written at once.  A worker's first and last item may
// be shared with its neighbours: those pieces (not normalised sum, maximum, sum of exponentials, all in fp32) go to two places per
// worker, and a second small launch joins them, always in the same order.  Items with a prefix to join leave theirs by row.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "dart_common.cuh"
#include "dart_shares.h"

namespace dart {
namespace attend {

constexpr float kLn2 = 0.69314718055994530942f;

// Division by a number that the host knows, for n < 2^31: a multiplication and a shift (Granlund and Montgomery's method: with
// 2^(s-1) < d <= 2^s and m = ceil(2^(32+s) / d) - 2^32, n / d = (mulhi(n, m) + n) >> s).  A division takes some thirty instructions, a
// 64-bit one is a call, and what a call of one token waits for is code that runs once.
struct Divisor {
    uint32_t m, s;
    __device__ __forceinline__ int of(int n) const { return (int)((__umulhi((uint32_t)n, m) + (uint32_t)n) >> s); }
};

// Partial results by row and head: [rows][Hq][D] and [rows][Hq] (maximum in log2 units, sum).
struct Whole {
    float *o;
    float2 *ml;
};

struct Open {
    int item, row0, n_q, hk, r0, len; // item < 0: none; its segment's rows and tokens, KV head, first row
    int pad[2];
};

// What one launch leaves for the joining one.
struct Pieces {
    int *item_base;  // [segments + 1] first item of every segment; the last: how many items, or -1: lengths that cannot be
    int2 *items;     // first and last worker of every item
    float *o;        // [workers][2][M][D]: a worker's first piece, and its last one where the item goes on at the next worker
    float2 *ml;      // [workers][2][M]
    Open *open;      // [workers] the item whose first piece, but not the last, is the worker's
    int M, n_workers; // rows of a tile
    Divisor by_M;
};

struct Params {
    const char *q;
    char *out;
    float *lse;
    long long q_stride, out_stride; // bytes
    const char *k, *v;
    int n_rows, Hq, Hk, R, n_seq, n_groups, n_pages, page_shift;
    int table_stride, ptable_stride;
    const int32_t *cu_q, *table, *kv_len, *cu_group, *ptable, *plen;
    Divisor by_R, by_Hk;
    float scale_log2;               // scale / ln 2: exponentials are powers of two
    int32_t *status;                // 4 words
    int n_prefix, n_own;            // segments of this launch: prefixes first
    int n_workers, max_items, least; // least: the most that a share's least size may be
    Pieces pieces;
    Whole whole[2];                 // [0] prefixes, [1] own tokens
};

struct Seg {
    int row0, n_q, len, nmb, width;
    const int32_t *table;
    bool prefix;
};

__device__ __forceinline__ int clamp(int x, int lo, int hi) { return min(max(x, lo), hi); }

// First packed row of sequence b.  (Offsets that do not ascend are held inside the rows: nothing out of bounds is touched.)
__device__ __forceinline__ int first_row(const Params &p, int b) { return p.cu_q ? clamp(p.cu_q[b], 0, p.n_rows) : b; }

// (kReport: the plan's first look at a segment, for all that come after it)
template <bool kReport = false>
__device__ inline Seg load_seg(const Params &p, int s)
{
    Seg g;
    int b0, b1;
    g.prefix = s < p.n_prefix;
    if (g.prefix) {
        b0 = clamp(p.cu_group[s], 0, p.n_seq), b1 = clamp(p.cu_group[s + 1], b0, p.n_seq);
        g.table = p.ptable + (long long)s * p.ptable_stride, g.width = p.ptable_stride, g.len = p.plen[s];
    } else {
        b0 = s - p.n_prefix, b1 = b0 + 1;
        g.table = p.table + (long long)b0 * p.table_stride, g.width = p.table_stride, g.len = p.kv_len[b0];
    }
    g.row0 = first_row(p, b0);
    g.n_q = max(first_row(p, b1) - g.row0, 0);
    const long long most = (long long)g.width << p.page_shift;
    if (g.len < 0 || g.len > most) {
        if (kReport) report_check(p.status);
        g.len = g.len < 0 ? 0 : (int)most;
    }
    g.nmb = g.prefix && g.len == 0 ? 0 : p.pieces.by_M.of(g.n_q * p.R + p.pieces.M - 1);
    return g;
}

// Whether a segment's offsets ascend inside what there is: others name rows twice (two workers would write them), or rows that are not there.
__device__ __forceinline__ bool ascends(const Params &p, int s)
{
    const int32_t *cu = s < p.n_prefix ? p.cu_group + s : p.cu_q + (s - p.n_prefix);
    return (s >= p.n_prefix && !p.cu_q) || (0 <= cu[0] && cu[0] <= cu[1] && cu[1] <= (s < p.n_prefix ? p.n_seq : p.n_rows));
}

// Own tokens that row t sees.
__device__ __forceinline__ int sees(const Seg &g, int t) { return g.prefix ? g.len : clamp(g.len - g.n_q + t + 1, 0, g.len); }
// ... and what the last row of a tile sees: how far its KV tiles go.  A sequence's rows have a tile even if they see nothing (it
// writes their zeros).
__device__ __forceinline__ int tile_sees(const Params &p, const Seg &g, int mb)
{
    return g.prefix ? g.len : sees(g, p.by_R.of(min((mb + 1) * p.pieces.M, g.n_q * p.R) - 1));
}
template <int kTile>
__device__ __forceinline__ int tiles_of(const Params &p, const Seg &g, int mb)
{
    return max(1, (tile_sees(p, g, mb) + kTile - 1) / kTile);
}
// A segment's part of the line.
template <int kTile, int kCost>
__device__ long long room_of(const Params &p, const Seg &g)
{
    if (g.nmb == 0) return 0;
    long long n = (long long)g.nmb * (kCost + tiles_of<kTile>(p, g, 0));
    if (!g.prefix && g.nmb > 1) {
        n = 0;
        for (int mb = 0; mb < g.nmb; ++mb) n += kCost + tiles_of<kTile>(p, g, mb);
    }
    return n * p.Hk;
}

// Where a worker begins, as the thread of the plan that comes by it leaves it.  (What a call of one token waits for is code that runs
// once, as fast as its instructions are fetched: everything here is kept short.)
struct Start {
    Seg g;
    int seg, item_base, hk, mb, from; // the item, and the place in its room
};

template <int kWorkers>
struct PlanShared {
    Start start[kWorkers];
    long long room[32], items[32];
    Shares share;
};

// Every CTA finds where its workers begin.  Block-wide; ends with a barrier.  (The line's length is counted in 32 bits, every row
// tile's KV tiles for themselves: a prompt of 2^21 rows and 32 heads in tiles of 256 x 128 would be 2^31.  Longer ones are reported.)
template <int kTile, int kCost, int kWorkers>
__device__ void plan(const Params &p, PlanShared<kWorkers> &sh)
{
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, nt = blockDim.x, n_seg = p.n_prefix + p.n_own;
    const int per = n_seg <= nt ? 1 : (n_seg + nt - 1) / nt, s0 = min(tid * per, n_seg), s1 = min(s0 + per, n_seg);
    long long items = 0, room = 0;
    Seg g;
#pragma unroll 1
    for (int s = s0; s < s1; ++s) {
        g = load_seg<true>(p, s);
        items += p.Hk * (long long)g.nmb, room += room_of<kTile, kCost>(p, g);
        if (!ascends(p, s)) room += 1ll << 32; // a line too long: reported, and nothing is done
    }
    long long i_sum = items, r_sum = room;
#pragma unroll 1
    for (int o = 1; o < 32; o <<= 1) {
        const long long a = __shfl_up_sync(0xffffffffu, i_sum, o), b = __shfl_up_sync(0xffffffffu, r_sum, o);
        if (lane >= o) i_sum += a, r_sum += b;
    }
    if (lane == 31) sh.items[warp] = i_sum, sh.room[warp] = r_sum;
    __syncthreads();
    long long i_all = 0, r_all = 0;
#pragma unroll 1
    for (int w = 0; w < nt / 32; ++w) {
        if (w == warp) i_sum += i_all, r_sum += r_all;
        i_all += sh.items[w], r_all += sh.room[w];
    }
    const bool ok = i_all <= p.max_items && r_all <= kLongestLine;
    const Shares share = Shares::of(ok ? (int)r_all : 0, i_all, p.n_workers, p.least);
    if (tid == 0) {
        sh.share = share;
        if (!ok) report_check(p.status);
    }
    if (ok && room > 0) {
        const int begin = (int)(r_sum - room), end = (int)r_sum; // the thread's part of the line
#pragma unroll 1
        for (int i = 0; i < kWorkers; ++i) {
            const int w = blockIdx.x * kWorkers + i, at = share.begin(w);
            if (at < begin || at >= end) continue;
            int base = (int)(i_sum - items), first = begin, s = s0;
            for (;; ++s) { // (with one segment a thread it is at hand)
                if (per > 1) g = load_seg(p, s);
                const int n = per > 1 ? (int)room_of<kTile, kCost>(p, g) : (int)room;
                if (at < first + n || s + 1 >= s1) {
                    const int head = p.by_Hk.of(n), off = at - first;
                    Start st;
                    st.g = g, st.seg = s, st.item_base = base;
                    st.hk = head > 0 ? (int)((unsigned)off / (unsigned)head) : 0;
                    st.from = off - st.hk * head;
                    for (st.mb = 0; st.mb < g.nmb - 1; ++st.mb) {
                        const int in = kCost + tiles_of<kTile>(p, g, st.mb);
                        if (st.from < in) break;
                        st.from -= in;
                    }
                    sh.start[i] = st;
                    break;
                }
                first += n, base += p.Hk * g.nmb;
            }
        }
    }
    if (blockIdx.x == 0) {
        int base = (int)(i_sum - items);
#pragma unroll 1
        for (int s = s0; s < s1; ++s) {
            p.pieces.item_base[s] = base;
            if (s + 1 < s1) base += p.Hk * load_seg(p, s).nmb;
        }
        if (tid == 0) p.pieces.item_base[n_seg] = ok ? (int)i_all : -1;
    }
    __syncthreads();
}

// A worker's way through its share of the line, piece by piece.
template <int kTile, int kCost>
struct Walk {
    Seg g;
    int s, item_base, hk, mb, a, b, nt, vis, worker; // piece: tiles [a, b) of nt
    int from, to;                                    // ... and its place in the item's room
    int left;
    bool done;

    template <int kWorkers>
    __device__ __forceinline__ void begin(const Params &p, const PlanShared<kWorkers> &sh, int local)
    {
        worker = blockIdx.x * kWorkers + local;
        left = sh.share.size(worker);
        done = left == 0;
        if (done) return;
        const Start &st = sh.start[local];
        g = st.g, s = st.seg, item_base = st.item_base, hk = st.hk, mb = st.mb, from = st.from;
        piece(p);
        if (a == b) next(p); // (a share that ends before the item's first tile)
    }
    __device__ __forceinline__ void piece(const Params &p)
    {
        vis = tile_sees(p, g, mb);
        nt = tiles_of<kTile>(p, g, mb);
        to = min(nt + kCost, from + left);
        a = max(0, from - kCost), b = max(0, to - kCost);
    }
    __device__ __forceinline__ void next(const Params &p)
    {
        do {
            left -= max(1, to - from);
            if (left <= 0) {
                done = true;
                return;
            }
            from = 0;
            if (++mb == g.nmb) {
                mb = 0;
                if (++hk == p.Hk) {
                    hk = 0;
                    do {
                        item_base += p.Hk * g.nmb;
                        if (++s >= p.n_prefix + p.n_own) {
                            done = true;
                            return;
                        }
                        g = load_seg(p, s);
                    } while (g.nmb == 0);
                }
            }
            piece(p);
        } while (a == b);
    }
    __device__ __forceinline__ int item() const { return item_base + hk * g.nmb + mb; }
    __device__ __forceinline__ bool is_whole() const { return a == 0 && b == nt; }
    __device__ __forceinline__ long long place() const { return 2ll * worker + (a == 0); }
    __device__ __forceinline__ void note(const Params &p) const // by one thread of the worker, once per piece
    {
        int *it = reinterpret_cast<int *>(p.pieces.items + item());
        if (a == 0) it[0] = worker;
        if (b == nt) it[1] = worker;
    }
};

// A worker's last piece, where the item goes on at the next worker: the joining launch starts from it.
__device__ __forceinline__ void no_open_item(const Params &p, int worker) { p.pieces.open[worker].item = -1; }
template <typename W>
__device__ __forceinline__ void open_item(const Params &p, const W &w)
{
    p.pieces.open[w.worker] = Open{w.item(), w.g.row0, w.g.n_q, w.hk, w.mb * p.pieces.M, w.g.len, {0, 0}};
}

// ---- types --------------------------------------------------------------------------------------------------------------
template <typename T>
__device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <>
__device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float lo, float hi)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}
template <>
__device__ __forceinline__ uint32_t pack2<__half>(float lo, float hi)
{
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ float exp2_approx(float x) // 2^x, within 2 ulp; 2^-inf = 0
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// A row's sum of exponentials is at least 1 where its scores are numbers (the largest weight is not below 1), NaN where one is NaN or
// +inf, and 0 where it sees nothing - or nothing but scores of -inf, of which there is no softmax either: that becomes NaN at the row's end.
__device__ __forceinline__ float settled(float l, bool sees_any) { return l == 0.0f && sees_any ? NAN : l; }
// what the sums are multiplied with; rows that see nothing are zeros
__device__ __forceinline__ float inverse(float l) { return l == 0.0f ? 0.0f : 1.0f / l; }
// log of the sum of exponentials, natural; -inf for rows that see nothing
__device__ __forceinline__ float lse_of(float m, float l) { return l == 0.0f ? -INFINITY : (m + log2f(l)) * kLn2; }

// ---- few rows -------------------------------------------------------------------------------------------------------------
// Tiles of 16 rows: bound by the cache's bytes, not by products, so that mma.sync (16 x 8 x 16) is enough.  Every WARP is a worker
// with a ring of its own in shared memory (cp.async, 16 bytes a lane; no barrier of the block, and nothing to merge between warps but
// what the joining launch merges anyway).  Keys and values of 32 tokens take turns in the ring; with three places of 8 KB and eight
// warps 128 KB are on their way per SM, which covers the latency of HBM at its full rate.  Tokens behind the end of a sequence
// are filled with zeros in shared memory, whatever their page holds: 0 * NaN would be NaN.
// Measured: 64 sequences of 164 to 676 tokens, 32 heads of 128, 88 us = 5.7 TB/s; two of 99000 and 131072 tokens, 4 KV heads, 85 us = 6.0 TB/s (copy
// rate 6.55).  Room of 0, 2, 4 tiles an item: 1, 1, 3 % slower; L2 prefetch hints on the copies: no difference.
constexpr int kNarrowM = 16, kNarrowTile = 32, kNarrowWarps = 8, kNarrowCost = 1, kNarrowLeast = 4;
constexpr int kNarrowRing = 24576; // bytes of a warp's ring

template <typename T>
__device__ __forceinline__ void mma_16816(float *c, const uint32_t *a, uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma_16816<__nv_bfloat16>(float *c, const uint32_t *a, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma_16816<__half>(float *c, const uint32_t *a, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <bool kTrans>
__device__ __forceinline__ void ldmatrix4(uint32_t *r, uint32_t addr)
{
    if (kTrans)
        asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
    else
        asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}

// A worker's loads, in the order in which they are consumed: keys, then values, of tile after tile.
template <int D>
struct Feed {
    Walk<kNarrowTile, kNarrowCost> w;
    int tile, pages, page_base; // tile at hand; lane l of `pages` holds table entry page_base + l
    bool values;

    __device__ __forceinline__ void fetch_pages(const Params &p, int from)
    {
        page_base = from;
        const int i = from + (threadIdx.x & 31), need = (w.vis + (1 << p.page_shift) - 1) >> p.page_shift;
        pages = -1;
        if (i < need) {
            pages = w.g.table[i];
            if (pages < 0 || pages >= p.n_pages) {
                pages = -1; // reads as zeros
                report_check(p.status);
            }
        }
    }
    __device__ __forceinline__ void enter(const Params &p)
    {
        tile = w.a, values = false;
        if (!w.done) fetch_pages(p, (tile * kNarrowTile) >> p.page_shift);
    }
    __device__ __forceinline__ void issue(const Params &p, uint32_t slot)
    {
        constexpr int kChunks = D / 8, kRowsPer = 32 / kChunks; // 16-byte chunks of a token; tokens per round of the warp
        if (!w.done) {
            const int lane = threadIdx.x & 31, tok0 = tile * kNarrowTile, chunk = lane % kChunks, mask = (1 << p.page_shift) - 1;
            if (!values && ((tok0 + kNarrowTile - 1) >> p.page_shift) >= page_base + 32) fetch_pages(p, tok0 >> p.page_shift);
            const char *base = values ? p.v : p.k;
            const int pg0 = __shfl_sync(0xffffffffu, pages, (tok0 >> p.page_shift) - page_base);
            const int pg1 = __shfl_sync(0xffffffffu, pages, ((tok0 + 16) >> p.page_shift) - page_base);
#pragma unroll
            for (int j = 0; j < kNarrowTile / kRowsPer; ++j) {
                const int t = j * kRowsPer + lane / kChunks, pg = t < 16 ? pg0 : pg1;
                const bool real = tok0 + t < w.vis && pg >= 0;
                const long long row = (((long long)(real ? pg : 0) * p.Hk + w.hk) << p.page_shift) + ((tok0 + t) & mask);
                const char *src = base + row * (D * 2) + chunk * 16;
                const uint32_t dst = slot + t * (D * 2) + ((chunk ^ (t & 7)) << 4);
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(real ? 16 : 0) : "memory");
            }
            if (values && ++tile == w.b) {
                w.next(p);
                enter(p);
            } else {
                values = !values;
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
};

template <typename T, int D>
__global__ void __launch_bounds__(kNarrowWarps * 32, 1) attend_narrow_kernel(const Params p)
{
    constexpr int kSlotBytes = kNarrowTile * D * 2, kSlots = kNarrowRing / kSlotBytes, kK = D / 16, kN = D / 8;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ PlanShared<kNarrowWarps> sh;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + warp * kNarrowRing;
    wait_for_previous();
    plan<kNarrowTile, kNarrowCost, kNarrowWarps>(p, sh);

    Walk<kNarrowTile, kNarrowCost> w;
    w.begin(p, sh, warp);
    if (lane == 0) no_open_item(p, w.worker);
    Feed<D> feed;
    feed.w = w;
    feed.enter(p);
#pragma unroll 1
    for (int i = 0; i < kSlots; ++i) feed.issue(p, ring + i * kSlotBytes);
    int slot = 0;
    // wait for the oldest load; afterwards its place is refilled
    const auto arrived = [&]() {
        asm volatile("cp.async.wait_group %0;" ::"n"(kSlots - 1) : "memory");
        __syncwarp();
        return ring + slot * kSlotBytes;
    };
    const auto refill = [&]() {
        __syncwarp();
        feed.issue(p, ring + slot * kSlotBytes);
        slot = slot + 1 == kSlots ? 0 : slot + 1;
    };

    for (; !w.done; w.next(p)) {
        const int rows = min(kNarrowM, w.g.n_q * p.R - w.mb * kNarrowM); // of this tile
        const int r0 = lane >> 2, r1 = r0 + 8, c0 = (lane & 3) * 2;
        // query fragments, and how many tokens the thread's two rows see
        uint32_t qa[kK][4];
        int lim[2];
        int row_n[2], row_h[2]; // packed row, head
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int r = w.mb * kNarrowM + (i ? r1 : r0);
            const bool real = (i ? r1 : r0) < rows;
            const int t = real ? p.by_R.of(r) : 0, h = w.hk * p.R + (real ? r - t * p.R : 0);
            lim[i] = real ? sees(w.g, t) : w.vis;
            row_n[i] = w.g.row0 + t, row_h[i] = h;
            const uint32_t *q = reinterpret_cast<const uint32_t *>(p.q + (long long)(w.g.row0 + t) * p.q_stride + (long long)h * (D * 2)) + (c0 >> 1);
#pragma unroll
            for (int kk = 0; kk < kK; ++kk) {
                qa[kk][i] = real ? q[kk * 8] : 0u;
                qa[kk][2 + i] = real ? q[kk * 8 + 4] : 0u;
            }
        }
        float o[kN][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f};
#pragma unroll
        for (int n = 0; n < kN; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.0f;

        for (int tile = w.a; tile < w.b; ++tile) {
            // scores of 32 tokens: four products of 8 tokens, two fragments of keys per ldmatrix
            uint32_t at = arrived();
            float s[4][4];
#pragma unroll
            for (int n = 0; n < 4; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.0f;
#pragma unroll
            for (int kk = 0; kk < kK; ++kk)
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    const int t = n * 16 + ((lane >> 4) << 3) + (lane & 7), chunk = 2 * kk + ((lane >> 3) & 1);
                    uint32_t b[4];
                    ldmatrix4<false>(b, at + t * (D * 2) + ((chunk ^ (t & 7)) << 4));
                    mma_16816<T>(s[2 * n], qa[kk], b[0], b[1]);
                    mma_16816<T>(s[2 * n + 1], qa[kk], b[2], b[3]);
                }
            refill();
            const int tok0 = tile * kNarrowTile + c0;
            const bool masked = __any_sync(0xffffffffu, min(lim[0], lim[1]) < (tile + 1) * kNarrowTile);
            float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
            for (int n = 0; n < 4; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s[n][i] *= p.scale_log2;
                    if (masked && tok0 + n * 8 + (i & 1) >= lim[i >> 1]) s[n][i] = -INFINITY;
                    top[i >> 1] = fmaxf(top[i >> 1], s[n][i]);
                }
            float fix[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 1));
                top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 2));
                const float now = fmaxf(m[i], top[i]);
                fix[i] = m[i] == now ? 1.0f : exp2_approx(m[i] - now); // (both -inf: 1)
                m[i] = now;
                top[i] = now == -INFINITY ? 0.0f : now;
                l[i] *= fix[i];
            }
            uint32_t pa[2][4];
#pragma unroll
            for (int n = 0; n < 4; ++n) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s[n][i] = exp2_approx(s[n][i] - top[i >> 1]);
                    l[i >> 1] += s[n][i];
                }
                // (weights enter the second product in the cache's type: half a step of it, relative, per token; fp16 weights below 2^-14 by
                // 2^-25 of the row's largest so far, those below that not at all, while the sum counts them: some 2^-25 of |v| each)
                pa[n >> 1][(n & 1) * 2] = pack2<T>(s[n][0], s[n][1]);
                pa[n >> 1][(n & 1) * 2 + 1] = pack2<T>(s[n][2], s[n][3]);
            }
            if (__any_sync(0xffffffffu, fix[0] != 1.0f || fix[1] != 1.0f))
#pragma unroll
                for (int n = 0; n < kN; ++n) o[n][0] *= fix[0], o[n][1] *= fix[0], o[n][2] *= fix[1], o[n][3] *= fix[1];
            at = arrived();
#pragma unroll
            for (int kk = 0; kk < 2; ++kk)
#pragma unroll
                for (int n = 0; n < kN / 2; ++n) {
                    const int t = kk * 16 + (((lane >> 3) & 1) << 3) + (lane & 7), chunk = 2 * n + (lane >> 4);
                    uint32_t b[4];
                    ldmatrix4<true>(b, at + t * (D * 2) + ((chunk ^ (t & 7)) << 4));
                    mma_16816<T>(o[2 * n], pa[kk], b[0], b[1]);
                    mma_16816<T>(o[2 * n + 1], pa[kk], b[2], b[3]);
                }
            refill();
        }

        if (lane == 0) {
            w.note(p);
            if (w.a == 0 && w.b < w.nt) open_item(p, w);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
            l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
            const int r = i ? r1 : r0;
            if (r >= rows) continue;
            if (w.is_whole() && p.n_groups == 0) {
                l[i] = settled(l[i], lim[i] > 0);
                const float inv = inverse(l[i]);
                uint32_t *dst = reinterpret_cast<uint32_t *>(p.out + row_n[i] * p.out_stride + (long long)row_h[i] * (D * 2)) + (c0 >> 1);
#pragma unroll
                for (int d = 0; d < kN; ++d) dst[d * 4] = pack2<T>(o[d][2 * i] * inv, o[d][2 * i + 1] * inv);
                if (p.lse && (lane & 3) == 0) p.lse[(long long)row_n[i] * p.Hq + row_h[i]] = lse_of(m[i], l[i]);
            } else {
                float *dst;
                float2 *ml;
                if (w.is_whole()) {
                    const Whole &to = p.whole[w.g.prefix ? 0 : 1];
                    const long long at = (long long)row_n[i] * p.Hq + row_h[i];
                    dst = to.o + at * D, ml = to.ml + at;
                } else {
                    const long long at = w.place() * kNarrowM + r;
                    dst = p.pieces.o + at * D, ml = p.pieces.ml + at;
                }
#pragma unroll
                for (int d = 0; d < kN; ++d) *reinterpret_cast<float2 *>(dst + d * 8 + c0) = make_float2(o[d][2 * i], o[d][2 * i + 1]);
                if ((lane & 3) == 0) *ml = make_float2(m[i], l[i]);
            }
        }
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
}

// ---- joining ----------------------------------------------------------------------------------------------------------------
struct JoinParams {
    Params p;           // (row tables, outputs, whole)
    Pieces from[2];     // [0] prefixes, [1] own tokens
    int seg_off[2];     // first segment of the kind in its launch
    int n_seg[2];       // segments of that launch
};

// Columns of a row that a lane holds: D / 32 of them, side by side.
template <int D>
struct Lane {
    float v[D / 32];
    __device__ __forceinline__ void load(const float *row)
    {
        const int lane = threadIdx.x & 31;
        if (D == 128) {
            const float4 x = *reinterpret_cast<const float4 *>(row + lane * 4);
            v[0] = x.x, v[1] = x.y, v[2 % (D / 32)] = x.z, v[3 % (D / 32)] = x.w;
        } else {
            const float2 x = *reinterpret_cast<const float2 *>(row + lane * 2);
            v[0] = x.x, v[1] = x.y;
        }
    }
};
template <typename T, int D>
__device__ __forceinline__ void write_row(const Params &p, int n, int h, const float *acc, float top, float sum)
{
    const int lane = threadIdx.x & 31;
    const float inv = inverse(sum);
    uint32_t *dst = reinterpret_cast<uint32_t *>(p.out + (long long)n * p.out_stride + (long long)h * (D * 2)) + lane * (D / 64);
#pragma unroll
    for (int d = 0; d < D / 64; ++d) dst[d] = pack2<T>(acc[2 * d] * inv, acc[2 * d + 1] * inv);
    if (p.lse && lane == 0) p.lse[(long long)n * p.Hq + h] = lse_of(top, sum);
}

// Without prefixes: what there is to join are the items that were cut, at most one per worker that begins one it does not end.  A
// few CTAs per worker, a warp per row, two rows a warp.  (Looking at every row and head instead: 111 us for the 358000 of four prompts of 2980 tokens, of
// which nearly none is cut.)
constexpr int kCutRows = 16; // of a CTA
template <typename T, int D>
__global__ void __launch_bounds__(256) attend_join_cut_kernel(const Params p, const Pieces f)
{
    constexpr int kPer = D / 32;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, first = blockIdx.x;
    wait_for_previous();
    const Open o = f.open[first];
    if (o.item < 0) return;
    const int last = f.items[o.item].y;
    if (last <= first || last >= f.n_workers) return; // (a worker that gave up left its items unnoted)
    const int all = last - first + 1, rows = min(f.M, o.n_q * p.R - o.r0);
    for (int r = blockIdx.y * kCutRows + warp; r < min(rows, (int)(blockIdx.y + 1) * kCutRows); r += 8) {
        // the item's first piece is the last one of its worker, the others are the first ones of theirs
        const auto at = [&](int i) { return (2ll * (first + i) + (i == 0)) * f.M + r; };
        float top = -INFINITY;
        for (int i = lane; i < all; i += 32) {
            const float2 v = f.ml[at(i)];
            if (v.y != 0.0f) top = fmaxf(top, v.x);
        }
#pragma unroll
        for (int k = 16; k > 0; k >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, k));
        float acc[kPer] = {}, sum = 0.0f;
#pragma unroll 4
        for (int i = 0; i < all; ++i) {
            const float2 v = f.ml[at(i)];
            Lane<D> x;
            x.load(f.o + at(i) * D);
            if (v.y == 0.0f) continue;
            const float wgt = exp2_approx(v.x - top);
            sum += v.y * wgt;
#pragma unroll
            for (int d = 0; d < kPer; ++d) acc[d] += x.v[d] * wgt;
        }
        const int t = p.by_R.of(o.r0 + r);
        write_row<T, D>(p, o.row0 + t, o.hk * p.R + (o.r0 + r - t * p.R), acc, top, settled(sum, o.len - o.n_q + t + 1 > 0));
    }
}

// Whether packed row n, of sequence b, sees tokens of its own.  (A function apart, of numbers: hardly any row asks, and inside the kernel it costs
// every call's few rows some 1 us.)
__device__ __noinline__ bool sees_own(const int32_t *cu_q, const int32_t *kv_len, int n_rows, long long most, int b, int n)
{
    const int row0 = cu_q ? clamp(cu_q[b], 0, n_rows) : b, n_q = cu_q ? clamp(cu_q[b + 1], 0, n_rows) - row0 : 1;
    return (int)min((long long)kv_len[b], most) - n_q + (n - row0) + 1 > 0;
}

// Row by row: with prefixes, where nearly every row has two pieces, and for few rows, whose lists of pieces are long.  kWarps
// warps share a row and head, or (kWarps 1) a warp takes `heads` heads of a row (at most 32).
template <typename T, int D, int kWarps>
__global__ void __launch_bounds__(kWarps > 1 ? kWarps * 32 : 128) attend_join_rows_kernel(const JoinParams j, const int heads)
{
    constexpr int kPer = D / 32;
    __shared__ float s_o[kWarps][D], s_sum[kWarps];
    const Params &p = j.p;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, part = kWarps > 1 ? warp : 0;
    const unsigned id = kWarps > 1 ? blockIdx.x : blockIdx.x * 4 + warp, per_row = (unsigned)(p.Hq + heads - 1) / (unsigned)heads;
    wait_for_previous();
    const int n = (int)(id / per_row), h0 = (int)(id - n * per_row) * heads, nh = min(heads, p.Hq - h0);
    if (n >= p.n_rows) return;
    int b = n;
    if (p.cu_q) {
        if (n < p.cu_q[0] || n >= p.cu_q[p.n_seq]) return;
        int lo = 0, hi = p.n_seq;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (p.cu_q[mid] <= n)
                lo = mid;
            else
                hi = mid;
        }
        b = lo;
    }
    // the lane's head (lanes 0 .. nh - 1; the others look at the last one): its pieces of the prefix, and its own
    const int h = h0 + min(lane, nh - 1), hk = p.by_R.of(h);
    int cnt[2] = {0, 0}, first[2] = {0, 0}, row_in[2] = {0, 0}; // first < 0: one piece, by row
    bool here = true;
#pragma unroll
    for (int kind = 0; kind < 2; ++kind) {
        int s = b, row0;
        if (kind == 0) {
            if (p.n_groups == 0) continue;
            if (j.from[0].item_base[j.n_seg[0]] < 0) return;
            if (b < p.cu_group[0] || b >= p.cu_group[p.n_groups]) continue; // in no group
            int lo = 0, hi = p.n_groups;
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (p.cu_group[mid] <= b)
                    lo = mid;
                else
                    hi = mid;
            }
            s = lo;
            if (p.plen[s] <= 0) continue;
            row0 = first_row(p, clamp(p.cu_group[s], 0, p.n_seq));
        } else {
            row0 = first_row(p, b);
        }
        const Pieces &f = j.from[kind];
        const int seg = j.seg_off[kind] + s;
        if (f.item_base[j.n_seg[kind]] < 0) return;
        const int base = f.item_base[seg], nmb = p.by_Hk.of(f.item_base[seg + 1] - base);
        const int r = (n - row0) * p.R + (h - hk * p.R), mb = f.by_M.of(r);
        if (r < 0 || mb >= nmb) { // (offsets that do not ascend)
            here = false;
            continue;
        }
        const int2 c = f.items[base + hk * nmb + mb];
        if (c.x < 0 || c.y < c.x || c.y >= f.n_workers || (c.x == c.y && p.n_groups == 0)) // (a worker that gave up; written already)
            here = false;
        else if (c.x == c.y)
            cnt[kind] = 1, first[kind] = -1;
        else
            cnt[kind] = c.y - c.x + 1, first[kind] = c.x, row_in[kind] = r - mb * f.M;
    }
    // two pieces at most, all by row: maxima and sums of the warp's heads at once
    const bool simple = kWarps == 1 && __all_sync(0xffffffffu, here && (cnt[0] == 0 || first[0] < 0) && first[1] < 0);
    if (simple) {
        const long long at = (long long)n * p.Hq + h;
        const float2 none = make_float2(-INFINITY, 0.0f), a = cnt[0] ? p.whole[0].ml[at] : none, o = p.whole[1].ml[at];
        const float top = fmaxf(a.y != 0.0f ? a.x : -INFINITY, o.y != 0.0f ? o.x : -INFINITY);
        const float w0 = a.y != 0.0f ? exp2_approx(a.x - top) : 0.0f, w1 = o.y != 0.0f ? exp2_approx(o.x - top) : 0.0f;
        float sum = a.y * w0 + o.y * w1;
        if (sum == 0.0f) sum = settled(sum, cnt[0] > 0 || sees_own(p.cu_q, p.kv_len, p.n_rows, (long long)p.table_stride << p.page_shift, b, n));
#pragma unroll 4
        for (int i = 0; i < nh; ++i) {
            const long long row = ((long long)n * p.Hq + h0 + i) * D;
            const float u0 = __shfl_sync(0xffffffffu, w0, i), u1 = __shfl_sync(0xffffffffu, w1, i);
            Lane<D> x, y; // (asked for before the weights are known; where a weight is 0 they may hold anything, where it is NaN the sum is)
            x.load(p.whole[0].o + row), y.load(p.whole[1].o + row);
            float acc[kPer];
#pragma unroll
            for (int d = 0; d < kPer; ++d) acc[d] = (u0 > 0.0f ? x.v[d] * u0 : 0.0f) + (u1 > 0.0f ? y.v[d] * u1 : 0.0f);
            write_row<T, D>(p, n, h0 + i, acc, __shfl_sync(0xffffffffu, top, i), __shfl_sync(0xffffffffu, sum, i));
        }
        return;
    }
    for (int i = 0; i < nh; ++i) {
        if (!__shfl_sync(0xffffffffu, (int)here, i)) continue; // (kWarps > 1: the same in all of them)
        const int n0 = __shfl_sync(0xffffffffu, cnt[0], i), n1 = __shfl_sync(0xffffffffu, cnt[1], i);
        const int f0 = __shfl_sync(0xffffffffu, first[0], i), f1 = __shfl_sync(0xffffffffu, first[1], i);
        const int r0 = __shfl_sync(0xffffffffu, row_in[0], i), r1 = __shfl_sync(0xffffffffu, row_in[1], i);
        const int all = n0 + n1;
        const auto find = [&](int k, const float *&o, const float2 *&ml) { // first the prefix's pieces, then its own
            const int kind = k < n0 ? 0 : 1, from = kind ? f1 : f0, at_row = kind ? r1 : r0;
            if (kind) k -= n0;
            const bool by_row = from < 0;
            // (an item's first piece is the last one of its worker, the others are the first ones of theirs)
            const long long at = by_row ? (long long)n * p.Hq + h0 + i : (2ll * (from + k) + (k == 0)) * j.from[kind].M + at_row;
            o = (by_row ? p.whole[kind].o : j.from[kind].o) + at * D, ml = (by_row ? p.whole[kind].ml : j.from[kind].ml) + at;
        };
        float top = -INFINITY;
        for (int k = lane; k < all; k += 32) {
            const float *o;
            const float2 *ml;
            find(k, o, ml);
            const float2 v = *ml;
            if (v.y != 0.0f) top = fmaxf(top, v.x);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        float acc[kPer] = {}, sum = 0.0f;
#pragma unroll 4
        for (int k = part; k < all; k += kWarps) {
            const float *o;
            const float2 *ml;
            find(k, o, ml);
            const float2 v = *ml;
            Lane<D> x;
            x.load(o);
            if (v.y == 0.0f) continue; // (its sums were not written)
            const float wgt = exp2_approx(v.x - top);
            sum += v.y * wgt;
#pragma unroll
            for (int d = 0; d < kPer; ++d) acc[d] += x.v[d] * wgt;
        }
        if (kWarps > 1) {
#pragma unroll
            for (int d = 0; d < kPer; ++d) s_o[part][lane * kPer + d] = acc[d];
            if (lane == 0) s_sum[part] = sum;
            __syncthreads();
            if (part != 0) return;
#pragma unroll 4
            for (int w = 1; w < kWarps; ++w) {
#pragma unroll
                for (int d = 0; d < kPer; ++d) acc[d] += s_o[w][lane * kPer + d];
                sum += s_sum[w];
            }
        }
        if (sum == 0.0f) sum = settled(sum, n0 > 0 || sees_own(p.cu_q, p.kv_len, p.n_rows, (long long)p.table_stride << p.page_shift, b, n));
        write_row<T, D>(p, n, h0 + i, acc, top, sum);
    }
}

} // namespace attend
} // namespace dart
